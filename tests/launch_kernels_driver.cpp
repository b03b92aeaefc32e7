// Host-only driver that names the kernels which the operators around the linear layer launch: the runtime's registration and launch calls
// are defined here, so that every launch is only written down.  No GPU is needed or used, and no pointer is dereferenced.
// Reads calls from standard input, one per line, and prints for each its launches, "kernel | workgroups in x, in y, threads", then
// "= status".
//   norm_forward tokens d stream_fp32 gate        norm_backward tokens d stream_fp32 gate
//   act_forward tokens m n ld_n                   act_backward tokens m n ld_n act outputs       (outputs: 1 dx, 2 G, 4 dbias)
//   gated_forward tokens m n ld_n                 gated_backward tokens m n ld_n act outputs
//   head_forward tokens h vocab ld                head_backward tokens h vocab ld 0 outputs
//   kernels                                       (all that the library holds)
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
    std::printf("%s | %u %u %u\n", names()[host].c_str(), grid.x, grid.y, block.x);
    return 0;
}
extern "C" int hipGetLastError() { return 0; }

template <typename T>
static T* at(uintptr_t address) { return reinterpret_cast<T*>(address); }   // aligned, never dereferenced

static int call(const std::string& what, int64_t a, int64_t b, int64_t c, int64_t d, int64_t e, int64_t outputs) {
    uint16_t *x = at<uint16_t>(0x10000), *y = at<uint16_t>(0x20000), *z = at<uint16_t>(0x30000), *o = at<uint16_t>(0x40000),
             *p = at<uint16_t>(0x50000), *q = at<uint16_t>(0x60000);
    float *f = at<float>(0x70000), *g = at<float>(0x80000);
    const int8_t* W = at<int8_t>(0x90000);
    const int64_t* labels = at<int64_t>(0xA0000);
    void* ws = at<void>(0x100000);
    const size_t all = ~(size_t)0;
    if (what == "norm_forward") return qg_residual_norm_forward(x, y, f, f, (int)d, f, 1.f, 1e-6f, a, b, 0, (int)c, o, p, nullptr);
    if (what == "norm_backward")
        return qg_residual_norm_backward(x, y, z, y, f, f, (int)d, f, 1.f, 1e-6f, a, b, 0, (int)c, o, p, g, g, d == QG_GATE_NONE ? nullptr : g,
                                         ws, all, nullptr);
    if (what == "act_forward") return qg_int8_linear_act_forward(x, W, f, y, z, QG_ACT_GELU, a, b, c, d, 0, 256, o, p, nullptr);
    if (what == "act_backward")
        return qg_int8_linear_act_backward(x, y, z, W, f, (int)e, a, b, c, d, 0, 256, outputs & 1 ? o : nullptr, outputs & 2 ? p : nullptr,
                                           outputs & 4 ? g : nullptr, ws, all, nullptr);
    if (what == "gated_forward") return qg_int8_gated_forward(x, W, f, W, f, QG_ACT_SILU, a, b, c, d, 0, 256, o, p, q, nullptr);
    if (what == "gated_backward")
        return qg_int8_gated_backward(x, y, z, x, W, f, W, f, (int)e, a, b, c, d, 0, 256, outputs & 1 ? o : nullptr, outputs & 2 ? p : nullptr,
                                      outputs & 2 ? q : nullptr, ws, all, nullptr);
    if (what == "head_forward") return qg_head_loss_forward(x, y, labels, a, b, c, d, f, g, ws, all, nullptr);
    if (what == "head_backward")
        return qg_head_loss_backward(x, y, labels, f, g, a, b, c, d, outputs & 1 ? o : nullptr, outputs & 2 ? p : nullptr, ws, all, nullptr);
    return -1;
}

int main() {
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream in(line);
        std::string what;
        int64_t v[6] = {};
        in >> what;
        for (int64_t& one : v) in >> one;
        if (what == "kernels") {
            for (const auto& k : names()) std::printf("%s | 0 0 0\n", k.second.c_str());
            std::printf("= 0\n");
        } else {
            std::printf("= %d\n", call(what, v[0], v[1], v[2], v[3], v[4], v[5]));
        }
    }
}
