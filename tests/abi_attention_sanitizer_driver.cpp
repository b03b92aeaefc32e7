// Host-only driver for the AddressSanitizer / UBSan build of the library: the host code of the attention half of a decoder layer, its refusals and
// its way up to every launch (the runtime's launch call is defined here and launches nothing), over sizes from one to the limits and beyond.
// No GPU is needed or used, and no pointer is dereferenced but the host's own.  Prints "sanitizer driver ok" and exits 0 when every
// return code is the expected one; a sanitizer report ends the process with a non-zero status.
#include <climits>
#include <initializer_list>
#include <cstdio>
#include <cstdlib>

#include "qgalore.h"

struct Extent {   // the runtime's dim3
    uint32_t x, y, z;
};
extern "C" unsigned __hipPushCallConfiguration(Extent, Extent, size_t, void*) { return 1; }   // (not zero: the kernel's stub is not called)
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
    const int32_t* const I = reinterpret_cast<const int32_t*>(0x30000);
    const int64_t* const P = reinterpret_cast<const int64_t*>(0x40000);
    const double* const W = reinterpret_cast<const double*>(0x50000);
    void* const S = reinterpret_cast<void*>(0x60000);
    const qg_heads x = {H, 1024, 64}, y = {H + 4096, (1 << 23) - 8, (int64_t(1) << 40) - 8};

    // attention: sizes to the limits, each option there and missing
    const int64_t tokens[] = {1, 63, 64, 1000, 8192, 100000, (1 << 24) - 1};
    for (int64_t q : tokens)
        for (int64_t k : tokens)
            for (int heads : {1, 12, 60})
                for (int sequences : {1, 17, 1 << 14})
                    for (int how = 0; how < 16; ++how) {
                        qg_attention a = {q, k, heads, heads % 3 ? 1 : heads / 3, 8 + 8 * (how % 16), sequences, I, I, how & 1 ? I : nullptr, how & 2 ? F : nullptr,
                                          0.1f, how & 4 ? 30.f : 0.f, 1, how & 1 ? 0 : how & 8 ? INT64_MAX : 0};
                        const size_t f = qg_attention_forward_workspace_bytes(&a), b = qg_attention_backward_workspace_bytes(&a);
                        EXPECT(qg_attention_forward(&a, &x, &y, &x, &y, how & 2 ? F : nullptr, S, f, nullptr), QG_OK);
                        EXPECT(qg_attention_backward(&a, &x, &y, &x, &y, &x, F, &x, &y, &x, S, b, nullptr), QG_OK);
                        EXPECT(qg_attention_backward(&a, &x, &y, &x, &y, &x, F, &x, &y, &x, S, b - 1, nullptr), QG_ERR_WORKSPACE);
                        if (f) EXPECT(qg_attention_forward(&a, &x, &y, &x, &y, F, nullptr, 0, nullptr), QG_ERR_WORKSPACE);
                    }
    qg_attention wild = {INT64_MAX, INT64_MIN, INT_MAX, INT_MIN, INT_MAX, INT_MAX, I, I, I, F, 1.f, 0.f, 1, INT64_MIN};
    EXPECT(qg_attention_forward(&wild, &x, &x, &x, &x, F, S, 0, nullptr), QG_ERR_SHAPE);
    wild.tokens_q = wild.tokens_k = 5;
    EXPECT(qg_attention_backward_workspace_bytes(&wild), 0);
    wild.heads_q = INT_MIN, wild.heads_k = -1;
    EXPECT(qg_attention_forward_workspace_bytes(&wild), 0);
    const qg_heads far = {H, INT64_MAX, INT64_MAX}, back = {H, INT64_MIN, 8};
    qg_attention plain = {100, 100, 8, 8, 64, 1, nullptr, nullptr, nullptr, nullptr, 0.125f, 0.f, 0, 0};
    EXPECT(qg_attention_forward(&plain, &far, &x, &x, &x, F, nullptr, 0, nullptr), QG_ERR_SHAPE);
    EXPECT(qg_attention_forward(&plain, &x, &back, &x, &x, F, nullptr, 0, nullptr), QG_ERR_SHAPE);
    EXPECT(qg_attention_forward(&plain, &x, &x, &x, &x, nullptr, nullptr, 0, nullptr), QG_OK);

    // rope and the cache
    for (int64_t t : tokens)
        for (int d : {8, 64, 96, 1024})
            for (int rot = 2; rot <= d; rot += d / 4)
                for (int layout = 0; layout < 2; ++layout) {
                    EXPECT(qg_rope_forward(&x, 12, nullptr, 0, P, W, t, d, rot, layout, 1.f, &x, nullptr, nullptr), QG_OK);
                    EXPECT(qg_rope_backward(&x, 1024, &x, 1024, P, W, t, d, rot, layout, -1.f, &y, &y, nullptr), QG_OK);
                    const qg_cache c = {H, H, I, 1000, 16, 4, d, 100, 50};
                    EXPECT(qg_cache_append(&c, nullptr, 0, &x, &x, P, nullptr, t, nullptr, 0, layout, 1.f, nullptr, nullptr), QG_OK);
                    EXPECT(qg_cache_append(&c, &x, 64, &x, &y, P, I, t, W, rot, layout, 1.f, &y, nullptr), QG_OK);
                }
    EXPECT(qg_rope_forward(&x, INT_MAX, &x, INT_MIN, P, W, 1, 64, 64, 0, 1.f, &x, &x, nullptr), QG_ERR_SHAPE);
    EXPECT(qg_rope_forward(&x, 1, &x, 1, P, W, INT64_MIN, INT_MIN, INT_MIN, INT_MIN, 1.f, &x, &x, nullptr), QG_ERR_SHAPE);
    double* out = static_cast<double*>(std::malloc(8 * 512));
    EXPECT(qg_rope_frequencies(1024, 10000.0, 8.0, 4096.0, 1.0, 4.0, out), QG_OK);
    EXPECT(qg_rope_frequencies(2, 1e-300, 1e300, 1e300, 0.0, 1e-300, out), QG_OK);
    EXPECT(qg_rope_frequencies(INT_MAX, 10000.0, 8.0, 0.0, 1.0, 4.0, out), QG_ERR_SHAPE);
    EXPECT(qg_rope_frequencies(INT_MIN, 10000.0, 8.0, 0.0, 1.0, 4.0, out), QG_ERR_SHAPE);
    std::free(out);
    for (int64_t sequences : {int64_t(1), int64_t(100), int64_t(1) << 20})
        for (int heads : {1, 8})
            for (int group : {1, 5, 17})
                for (int width : {1, 100, 1 << 10})
                    for (int page : {1, 16, 1000}) {
                        const qg_cache c = {H, H, I, 1000, page, heads, 128, (int)sequences, width};
                        const bool fits = sequences * heads * group < (1 << 24) && sequences * width < (int64_t(1) << 31);
                        const size_t n = qg_attention_paged_workspace_bytes(&c, heads * group);
                        EXPECT(n != 0, fits);
                        if (!fits) continue;
                        EXPECT(qg_attention_paged(&c, I, &x, heads * group, 0.1f, 0.f, INT64_MAX, nullptr, &y, S, n, nullptr), QG_OK);
                        EXPECT(qg_attention_paged(&c, I, &x, heads * group, 0.1f, 30.f, 10, F, &y, S, n - 1, nullptr), QG_ERR_WORKSPACE);
                    }
    const qg_cache huge = {H, H, I, INT64_MAX, INT_MAX, INT_MAX, INT_MAX, INT_MAX, INT_MAX}, less = {H, H, I, INT64_MIN, INT_MIN, INT_MIN, INT_MIN, INT_MIN, INT_MIN};
    for (const qg_cache* c : {&huge, &less}) {
        EXPECT(qg_attention_paged_workspace_bytes(c, INT_MAX), 0);
        EXPECT(qg_cache_append(c, &x, 1, &x, &x, P, I, 1, W, 2, 0, 1.f, &x, nullptr), QG_ERR_SHAPE);
    }
    const qg_cache most = {H, H, I, INT64_MAX, 2, 1, 64, 1, 1};
    EXPECT(qg_attention_paged_workspace_bytes(&most, 1), 0);
    if (failures == 0) std::printf("sanitizer driver ok\n");
    return failures != 0;
}
