// Host-only driver for the launch geometry of the operators around the linear layer, as launch_geometry_driver.cpp is for the rest: the
// runtime's launch call is defined here and launches nothing, so that every grid is only looked at.  No GPU is needed or used,
// and no pointer is dereferenced.
//   norm_forward tokens d        norm_backward tokens d
//   act_forward tokens m n       act_backward tokens m n        gated_forward ...        gated_backward ...
//   head_forward tokens h vocab  head_backward tokens h vocab
// Prints each launch as "workgroups in x, in y, threads"; exits 1 if one exceeds what the runtime accepts: fewer than 2^32 threads in
// x, 65535 workgroups in y and in z, none of them zero.
#include <cstdio>
#include <cstdlib>
#include <string>

#include "qgalore.h"

static long launches = 0, refused = 0;

struct Extent {   // the runtime's dim3
    uint32_t x, y, z;
};

extern "C" unsigned __hipPushCallConfiguration(Extent grid, Extent block, size_t, void*) {
    ++launches;
    const uint64_t x = (uint64_t)grid.x * block.x;
    if (x == 0 || x >> 32 != 0 || grid.y == 0 || grid.y > 65535 || grid.z == 0 || grid.z > 65535) {
        if (refused++ == 0) std::printf("refused: grid %u x %u x %u of %u threads\n", grid.x, grid.y, grid.z, block.x);
    }
    std::printf("%u %u %u\n", grid.x, grid.y, block.x);
    return 1;   // (not zero: the kernel's stub is not called)
}
extern "C" int hipGetLastError() { return 0; }

template <typename T>
static T* at(uintptr_t address) { return reinterpret_cast<T*>(address); }   // aligned, never dereferenced

int main(int argc, char** argv) {
    if (argc < 4) return 2;
    const std::string what = argv[1];
    const int64_t a = std::atoll(argv[2]), b = std::atoll(argv[3]), c = argc > 4 ? std::atoll(argv[4]) : 0;
    uint16_t *x = at<uint16_t>(0x10000), *y = at<uint16_t>(0x20000), *z = at<uint16_t>(0x30000), *o = at<uint16_t>(0x40000),
             *p = at<uint16_t>(0x50000), *q = at<uint16_t>(0x60000);
    float *f = at<float>(0x70000), *g = at<float>(0x80000);
    const int8_t* W = at<int8_t>(0x90000);
    const int64_t* labels = at<int64_t>(0xA0000);
    void* ws = at<void>(0x100000);
    const size_t all = ~(size_t)0;
    int status = -1;
    if (what == "norm_forward")
        status = qg_residual_norm_forward(x, y, f, f, QG_GATE_CHANNEL, f, 1.f, 1e-6f, a, b, 0, 0, o, p, nullptr);
    else if (what == "norm_backward")
        status = qg_residual_norm_backward(x, y, z, y, f, f, QG_GATE_CHANNEL, f, 1.f, 1e-6f, a, b, 0, 0, o, p, g, g, g, ws,
                                           qg_residual_norm_workspace_bytes(a, b), nullptr);
    else if (what == "act_forward")
        status = qg_int8_linear_act_forward(x, W, f, y, z, QG_ACT_GELU, a, b, c, 0, 0, 256, o, p, nullptr);
    else if (what == "act_backward")
        status = qg_int8_linear_act_backward(x, y, z, W, f, QG_ACT_GELU, a, b, c, 0, 0, 256, o, p, g, ws,
                                             qg_int8_linear_act_workspace_bytes(a, b, c), nullptr);
    else if (what == "gated_forward")
        status = qg_int8_gated_forward(x, W, f, W, f, QG_ACT_SILU, a, b, c, 0, 0, 256, o, p, q, nullptr);
    else if (what == "gated_backward")
        status = qg_int8_gated_backward(x, y, z, x, W, f, W, f, QG_ACT_SILU, a, b, c, 0, 0, 256, o, p, q, ws,
                                        qg_int8_gated_workspace_bytes(a, b, c), nullptr);
    else if (what == "head_forward")
        status = qg_head_loss_forward(x, y, labels, a, b, c, 0, f, g, ws, all, nullptr);
    else if (what == "head_backward")
        status = qg_head_loss_backward(x, y, labels, f, g, a, b, c, 0, o, p, ws, all, nullptr);
    std::printf("status %d, %ld launches, %ld refused\n", status, launches, refused);
    return status != QG_OK || refused != 0 || launches == 0;
}
