// Host-only driver for the attention half of a decoder layer: the runtime's registration and launch calls are defined here, so that every launch is
// only written down and looked at.  No GPU is needed or used, and no pointer is dereferenced.  Reads calls from standard input, one per
// line, and prints for each its launches, "kernel | workgroups in x, threads", then "= status"; a grid that the runtime would not accept (2^32
// threads or more, none) gives status 1000.
//   rope tokens heads_q heads_k d rot layout out_of_place          append tokens heads_q heads_k d rot layout page_size
//   forward tokens_q tokens_k heads_q heads_k d sequences flags    backward ... (flags: 1 causal, 2 cap, 4 slopes, 8 window, 16 prefix)
//   paged sequences heads_q heads_k d page_size width flags        kernels (all that the library holds)
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <iostream>
#include <map>
#include <sstream>
#include <string>

#include "qgalore.h"

struct Extent {   // the runtime's dim3
    uint32_t x, y, z;
};
static Extent grid_now, block_now;
static bool refused = false;

static std::map<const void*, std::string>& names() {   // (filled by the library's constructors, ahead of main)
    static std::map<const void*, std::string> all;
    return all;
}
static std::string readable(const char* mangled) {
    int status = 0;
    char* s = abi::__cxa_demangle(mangled, nullptr, nullptr, &status);
    std::string out = status == 0 ? s : mangled;
    std::free(s);
    return out.substr(0, out.find('('));
}

extern "C" void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, Extent*, Extent*, int*) {
    names()[host] = readable(device);
}
extern "C" unsigned __hipPushCallConfiguration(Extent grid, Extent block, size_t, void*) {
    grid_now = grid;
    block_now = block;
    return 0;
}
extern "C" unsigned __hipPopCallConfiguration(Extent* grid, Extent* block, size_t* shared, void** stream) {
    *grid = grid_now;
    *block = block_now;
    *shared = 0;
    *stream = nullptr;
    return 0;
}
extern "C" int hipLaunchKernel(const void* host, Extent grid, Extent block, void**, size_t, void*) {
    const uint64_t threads = (uint64_t)grid.x * block.x;
    refused |= threads == 0 || threads >> 32 != 0 || grid.y != 1 || grid.z != 1;
    std::printf("%s | %u %u\n", names()[host].c_str(), grid.x, block.x);
    return 0;
}
extern "C" int hipGetLastError() { return 0; }

template <typename T>
static T* at(uintptr_t address) { return reinterpret_cast<T*>(address); }   // aligned, never dereferenced

static int call(const std::string& what, const int64_t* v) {
    const qg_heads x = {at<uint16_t>(0x10000), 1 << 12, 1 << 10}, y = {at<uint16_t>(0x20000), 1 << 12, 1 << 10};
    const int64_t* positions = at<int64_t>(0x30000);
    const double* freqs = at<double>(0x40000);
    const int32_t* ints = at<int32_t>(0x50000);
    float* f = at<float>(0x60000);
    void* ws = at<void>(0x100000);
    const size_t all = ~(size_t)0;
    if (what == "rope") {
        const qg_heads& out = v[6] ? y : x;
        int e = qg_rope_forward(&x, (int)v[1], &x, (int)v[2], positions, freqs, v[0], (int)v[3], (int)v[4], (int)v[5], 1.f, &out, &out, nullptr);
        return e ? e : qg_rope_backward(&x, (int)v[1], &x, (int)v[2], positions, freqs, v[0], (int)v[3], (int)v[4], (int)v[5], 1.f, &out, &out, nullptr);
    }
    if (what == "append") {
        const qg_cache c = {at<uint16_t>(0x70000), at<uint16_t>(0x80000), ints, 1000, (int)v[6], (int)v[2], (int)v[3], 64, 100};
        return qg_cache_append(&c, &x, (int)v[1], &x, &x, positions, ints, v[0], freqs, (int)v[4], (int)v[5], 1.f, &y, nullptr);
    }
    if (what == "forward" || what == "backward") {
        const int64_t flags = v[6];
        qg_attention a = {v[0], v[1], (int)v[2], (int)v[3], (int)v[4], (int)v[5], ints, v[0] == v[1] ? nullptr : ints, flags & 16 ? ints : nullptr,
                          flags & 4 ? f : nullptr, 0.125f, flags & 2 ? 20.f : 0.f, (int)(flags & 1), flags & 8 ? 100 : 0};
        if (what == "forward") return qg_attention_forward(&a, &x, &x, &x, &y, f, ws, qg_attention_forward_workspace_bytes(&a), nullptr);
        return qg_attention_backward(&a, &x, &x, &x, &x, &x, f, &y, &y, &y, ws, qg_attention_backward_workspace_bytes(&a), nullptr);
    }
    if (what == "paged") {
        const qg_cache c = {at<uint16_t>(0x70000), at<uint16_t>(0x80000), ints, 1000, (int)v[4], (int)v[2], (int)v[3], (int)v[0], (int)v[5]};
        return qg_attention_paged(&c, ints, &x, (int)v[1], 0.125f, v[6] & 2 ? 20.f : 0.f, 0, v[6] & 4 ? f : nullptr, &y, ws, all, nullptr);
    }
    return -1;
}

int main() {
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream in(line);
        std::string what;
        int64_t v[8] = {};
        in >> what;
        for (int64_t& one : v) in >> one;
        if (what == "kernels") {
            for (const auto& k : names()) std::printf("%s | 0 0\n", k.second.c_str());
            std::printf("= 0\n");
        } else {
            refused = false;
            const int status = call(what, v);
            std::printf("= %d\n", refused ? 1000 : status);
        }
    }
}
