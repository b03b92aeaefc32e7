// Host-only driver for the AddressSanitizer / UBSan build of the library: the host code of the operators around the linear layer, its refusals
// and its way up to every launch (the runtime's launch call is defined here and launches nothing), with every optional argument there
// and missing, over sizes from one to the limits.  No GPU is needed or used, and no pointer is dereferenced.  Prints "sanitizer
// driver ok" and exits 0 when every return code is the expected one; a sanitizer report ends the process with a non-zero status.
#include <cstdio>
#include <initializer_list>

#include "qgalore.h"

struct Extent {   // the runtime's dim3
    uint32_t x, y, z;
};
static long launches = 0;
extern "C" unsigned __hipPushCallConfiguration(Extent, Extent, size_t, void*) {
    ++launches;
    return 1;   // (not zero: the kernel's stub is not called)
}
extern "C" int hipGetLastError() { return 0; }

static int failures = 0;
#define EXPECT(call, want)                                                              \
    do {                                                                                \
        const long long got_ = (long long)(call);                                       \
        if (got_ != (long long)(want)) {                                                \
            std::printf("line %d: %s = %lld, expected %lld\n", __LINE__, #call, got_, (long long)(want)); \
            ++failures;                                                                 \
        }                                                                               \
    } while (0)

int main() {
    uint16_t* const H = reinterpret_cast<uint16_t*>(0x10000);
    float* const F = reinterpret_cast<float*>(0x20000);
    int8_t* const Q = reinterpret_cast<int8_t*>(0x30000);
    int64_t* const L = reinterpret_cast<int64_t*>(0x40000);
    void* const S = reinterpret_cast<void*>(0x50000);
    const size_t all = ~(size_t)0;
    const int64_t lim = int64_t(1) << 31;

    // norms: each side there and missing
    const int64_t norms[][2] = {{1, 1}, {3, 512}, {1000, 2047}, {8192, 4096}, {5, 8192}, {7, 16384}, {(1 << 22) - 1, 1}, {(1 << 22) - 1, 16384}};
    for (auto& s : norms)
        for (int fp32 = 0; fp32 < 2; ++fp32)
            for (int gate = 0; gate < 3; ++gate)
                for (int parts = 1; parts < 4; ++parts) {
                    uint16_t *y = parts & 1 ? H : nullptr, *u = parts & 2 ? H : nullptr;
                    EXPECT(qg_residual_norm_forward(H, y, nullptr, F, gate, F, 1.f, 0.f, s[0], s[1], 0, fp32, y ? H : nullptr, u, nullptr), QG_OK);
                    EXPECT(qg_residual_norm_backward(u, y, H, y, nullptr, F, gate, F, 1.f, 0.f, s[0], s[1], 0, fp32, H, y, nullptr, nullptr, nullptr,
                                                     nullptr, 0, nullptr), QG_OK);
                    const size_t bytes = qg_residual_norm_workspace_bytes(s[0], s[1]);
                    EXPECT(qg_residual_norm_backward(H, y, H, y, F, F, gate, F, 1.f, 1e-6f, s[0], s[1], 0, fp32, H, y, F, y ? F : nullptr,
                                                     y && gate ? F : nullptr, S, bytes, nullptr), QG_OK);
                }
    EXPECT(qg_residual_norm_workspace_bytes(INT64_MAX, INT64_MAX), 0);
    EXPECT(qg_residual_norm_workspace_bytes(-1, 4), 0);
    EXPECT(qg_residual_norm_forward(H, H, F, nullptr, 0, F, 1.f, 1e-6f, INT64_MIN, 512, 0, 0, H, H, nullptr), QG_ERR_SHAPE);
    EXPECT(qg_residual_norm_forward(H, H, F, nullptr, 0, F, 1.f, 1e-6f, 16, 512, INT64_MAX, 0, H, H, nullptr), QG_ERR_SHAPE);
    EXPECT(qg_residual_norm_backward(H, H, H, H, F, F, 1, F, 1.f, 1e-6f, 16, 512, 0, 0, H, H, F, F, F, nullptr, 0, nullptr), QG_ERR_WORKSPACE);

    // linear layers: outputs by themselves and together, the workspace missing where it is not needed
    const int64_t layers[][3] = {{1, 1, 1}, {1, 11008, 4096}, {64, 4096, 4096}, {150, 4095, 2047}, {256, 2048, 768}, {500, 4096, 2048}, {1000, 2048, 5461},
                                 {1024, 4096, 1024}, {4096, 11008, 4096}, {4000, 11008, 4096}, {100, 5461, 1027}, {2049, 33, 70}, {32, 40000000, 32},
                                 {32, 32, 40000000}, {lim / 16 - 1, 8, 8}, {8, (1 << 27) - 1, 8}, {8, 8, (1 << 27) - 1}, {46340, 46340, 46340}};
    for (auto& s : layers) {
        const int64_t T = s[0], m = s[1], n = s[2];
        const size_t wa = qg_int8_linear_act_workspace_bytes(T, m, n), wg = qg_int8_gated_workspace_bytes(T, m, n);
        for (int act = QG_ACT_NONE; act <= QG_ACT_GELU; ++act) {
            EXPECT(qg_int8_linear_act_forward(H, Q, F, act & 1 ? H : nullptr, act & 2 ? H : nullptr, act, T, m, n, 0, 0, 256, act & 1 ? nullptr : H, H,
                                              nullptr), QG_OK);
            EXPECT(qg_int8_gated_forward(H, Q, F, Q, F, act, T, m, n, 0, 0, 256, act & 1 ? H : nullptr, act & 1 ? H : nullptr, H, nullptr), QG_OK);
            for (int out = 1; out < 8; ++out) {
                uint16_t *dx = out & 1 ? H : nullptr, *G = out & 2 ? H : nullptr;
                float* db = out & 4 ? F : nullptr;
                const bool space = act != QG_ACT_NONE || db;
                EXPECT(qg_int8_linear_act_backward(H, act == QG_ACT_NONE ? nullptr : H, G ? H : nullptr, dx ? Q : nullptr, dx ? F : nullptr, act, T, m, n,
                                                   0, 0, 256, dx, G, db, space ? S : nullptr, space ? wa : 0, nullptr), QG_OK);
                if (space)
                    EXPECT(qg_int8_linear_act_backward(H, H, H, Q, F, act, T, m, n, 0, 0, 256, dx, G, db, S, wa - 1, nullptr), QG_ERR_WORKSPACE);
                if (out < 4)
                    EXPECT(qg_int8_gated_backward(H, H, H, G ? H : nullptr, dx ? Q : nullptr, dx ? F : nullptr, dx ? Q : nullptr, dx ? F : nullptr, act,
                                                  T, m, n, 0, 0, 256, dx, G, G, S, wg, nullptr), QG_OK);
            }
        }
        EXPECT(qg_int8_gated_backward(H, H, H, H, Q, F, Q, F, 2, T, m, n, 0, 0, 256, H, H, H, S, wg - 1, nullptr), QG_ERR_WORKSPACE);
        EXPECT(qg_int8_gated_backward(H, H, H, H, Q, F, Q, F, 2, T, m, n, 0, 0, 256, H, H, H, nullptr, wg, nullptr), QG_ERR_WORKSPACE);
    }
    for (int64_t bad : {(int64_t)0, (int64_t)-1, INT64_MIN, INT64_MAX, lim}) {
        EXPECT(qg_int8_linear_act_workspace_bytes(bad, 4, 4), 0);
        EXPECT(qg_int8_gated_workspace_bytes(4, bad, 4), 0);
        EXPECT(qg_int8_linear_act_forward(H, Q, F, H, H, 1, 4, 4, bad, 0, 0, 256, H, H, nullptr), QG_ERR_SHAPE);
        EXPECT(qg_int8_gated_forward(H, Q, F, Q, F, 1, 4, bad, 4, 0, 0, 256, H, H, H, nullptr), QG_ERR_SHAPE);
        if (bad != 0) EXPECT(qg_int8_linear_act_forward(H, Q, F, H, H, 1, 4, 4, 4, bad, 0, 256, H, H, nullptr), QG_ERR_SHAPE);
        EXPECT(qg_head_loss_workspace_bytes(4, 4, bad), 0);
        EXPECT(qg_head_loss_forward(H, H, L, bad, 4, 4, 0, F, F, S, all, nullptr), QG_ERR_SHAPE);
        if (bad != 0) EXPECT(qg_head_loss_backward(H, H, L, F, F, 4, 4, 4, bad, H, H, S, all, nullptr), QG_ERR_SHAPE);
    }

    // the head: one gradient and both, around the sizes where tiles, pieces and parts change, up to the limits
    const int64_t heads[][3] = {{1, 1, 1}, {1, 768, 4001}, {64, 64, 64}, {65, 72, 600000}, {256, 768, 32000}, {1000, 2048, 32003}, {1000, 1100, 32003},
                                {1500, 1024, 9001}, {4096, 4096, 32000}, {4100, 4100, 1100}, {70000, 16, 300}, {(1 << 24) - 1, 1, 16383},
                                {(1 << 24) - 1, 1023, 16384}, {16383, 8191, (1 << 24) - 1}, {1, 8191, (1 << 24) - 1}, {1, 65535, (1 << 21) - 1},
                                {(1 << 18) - 1, 65535, 1}, {400000, 64, 600000}};
    for (auto& s : heads) {
        const size_t bytes = qg_head_loss_workspace_bytes(s[0], s[1], s[2]);
        EXPECT(bytes > 0, 1);
        EXPECT(qg_head_loss_forward(H, H, L, s[0], s[1], s[2], 0, F, F, S, bytes, nullptr), QG_OK);
        EXPECT(qg_head_loss_forward(H, H, L, s[0], s[1], s[2], 0, F, F, S, 64, nullptr), QG_ERR_WORKSPACE);
        for (int out = 1; out < 4; ++out)
            EXPECT(qg_head_loss_backward(H, H, L, F, F, s[0], s[1], s[2], 0, out & 1 ? H : nullptr, out & 2 ? H : nullptr, S, bytes, nullptr), QG_OK);
        EXPECT(qg_head_loss_backward(H, H, L, F, F, s[0], s[1], s[2], 0, H, H, nullptr, bytes, nullptr), QG_ERR_WORKSPACE);
    }

    if (failures || launches == 0) {
        std::printf("%d unexpected return codes, %ld launches\n", failures, launches);
        return 1;
    }
    std::printf("sanitizer driver ok\n");
    return 0;
}
