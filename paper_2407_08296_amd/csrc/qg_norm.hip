// Norms of the residual stream: what stands between two blocks of a decoder, in one pass over the stream.  For every token
//     n  = w_post * y / rms(y)                    the norm behind a block (optional), y the block's output
//     h' = h + scale * gate * n                   its gate (none, one per channel, or one per token and channel), and the sum
//     u  = w_pre * h' / rms(h')                   the norm ahead of the next block (optional);  rms(v) = sqrt(mean v^2 + eps)
// and the gradients: with r = 1/rms(h'), q = 1/rms(y), a = w_pre du, k = scale * gate * w_post,
//     dh = dh' + r (a - h' r^2 mean(a h'))        of h and h' alike
//     dy = q (k dh - y q^2 mean(k dh y))
//     dw_pre = sum_t du h' r,   dw_post = sum_t scale gate dh y q,   dgate = scale dh w_post y q (summed over t if per channel)
// Every array is read or written once; a row stays in the registers of one workgroup (or wave), and HBM is the bound.  Not so the backward
// pass of rows beyond 8192 elements: it spills, and is bound by that (see there).
#include "qg_common.h"
#include "qg_gemm_kernels.h"

namespace qg {

constexpr int kNormMaxD = 16384;
constexpr int64_t kNormMaxTokens = int64_t(1) << 22;   // (a workgroup of up to 1024 threads per token, 2^32 threads per launch)
enum : int { kGateNone = QG_GATE_NONE, kGateChannel = QG_GATE_CHANNEL, kGateToken = QG_GATE_TOKEN };

// 8 consecutive elements of a row, of which the first `valid` exist (the others read as 0); rows may start at any element.  Past
// the end the last element is read again: the loads of a row's end are independent of each other, where seven conditional ones
// would wait for one another (1000 rows of 2047, five arrays: 26 us of which the row ends took half).
__device__ __forceinline__ u32x4 load8_raw(const uint16_t* p, int valid) {
    if (valid >= 8) return *reinterpret_cast<const u32x4_align2*>(p);
    u32x4 w = {0u, 0u, 0u, 0u};
    if (valid > 0) {
        uint32_t e[7];
#pragma unroll
        for (int j = 0; j < 7; ++j) e[j] = p[min(j, valid - 1)];
#pragma unroll
        for (int j = 0; j < 7; ++j) w[j >> 1] |= j < valid ? e[j] << (16 * (j & 1)) : 0u;
    }
    return w;
}
__device__ __forceinline__ void load8(const uint16_t* p, int valid, float (&v)[8]) {
    const u32x4 w = load8_raw(p, valid);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __builtin_bit_cast(float, w[j] << 16);
        v[2 * j + 1] = __builtin_bit_cast(float, w[j] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, int valid, float (&v)[8]) {
    if (valid >= 8) {
        const u32x4 a = reinterpret_cast<const u32x4_align4*>(p)[0], b = reinterpret_cast<const u32x4_align4*>(p)[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = __builtin_bit_cast(float, (uint32_t)a[j]);
            v[4 + j] = __builtin_bit_cast(float, (uint32_t)b[j]);
        }
    } else {
        float e[7] = {};
        if (valid > 0)
#pragma unroll
            for (int j = 0; j < 7; ++j) e[j] = p[min(j, valid - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < valid ? e[min(j, 6)] : 0.f;
    }
}
__device__ __forceinline__ void store8(uint16_t* p, int valid, const float (&v)[8]) {
    const u32x4 w = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    if (valid >= 8) {
        *reinterpret_cast<u32x4_align2*>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < valid) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
}
__device__ __forceinline__ void store8(float* p, int valid, const float (&v)[8]) {
    if (valid >= 8) {
        u32x4 a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = __builtin_bit_cast(uint32_t, v[j]);
            b[j] = __builtin_bit_cast(uint32_t, v[4 + j]);
        }
        reinterpret_cast<u32x4_align4*>(p)[0] = a;
        reinterpret_cast<u32x4_align4*>(p)[1] = b;
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < valid) p[j] = v[j];
    }
}

// Sum over the 64 lanes, the same in each, without LDS: neighbours, quads and halves of 16 lanes by data-parallel moves, then the 16s
// and 32s swapped.
__device__ __forceinline__ float lanes_sum(float v) {
    auto moved = [&](auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    v += moved(std::integral_constant<int, 0xB1>());    // lane ^ 1
    v += moved(std::integral_constant<int, 0x4E>());    // lane ^ 2
    v += moved(std::integral_constant<int, 0x141>());   // the 8 lanes mirrored
    v += moved(std::integral_constant<int, 0x140>());   // the 16 lanes mirrored
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    v = __builtin_bit_cast(float, (uint32_t)s[0]) + __builtin_bit_cast(float, (uint32_t)s[1]);
    const uint32_t c = __builtin_bit_cast(uint32_t, v);
    const auto u = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return __builtin_bit_cast(float, (uint32_t)u[0]) + __builtin_bit_cast(float, (uint32_t)u[1]);
}

// Sums of N values over the WPR waves that share a row, the same value in every lane; `slot`: N floats of LDS per wave of the
// workgroup, another set than that of the call before.  A fixed order: the result does not depend on timing.
template <int N, int WPR>
__device__ __forceinline__ void row_sums(float (&s)[N], float* slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = lanes_sum(s[i]);
    if constexpr (WPR > 1) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave / WPR * WPR;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) slot[wave * N + i] = s[i];
        __syncthreads();
        // lane l takes wave l's sums, zero beyond the last; all lanes add
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = lanes_sum(lane < WPR ? slot[(first + min(lane, WPR - 1)) * N + i] : 0.f);
    }
}

// 8 elements as they come from memory, kept so between their two uses.
template <typename S>
struct Raw8 {
    u32x4 w[sizeof(S) / 2];
    __device__ __forceinline__ void load(const S* p, int valid) {
        if constexpr (sizeof(S) == 2) {
            w[0] = load8_raw(p, valid);
        } else if (valid >= 8) {
            w[0] = *reinterpret_cast<const u32x4_align4*>(p);
            w[1] = *reinterpret_cast<const u32x4_align4*>(p + 4);
        } else {
            float e[8];
            load8(p, valid, e);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j / 4][j % 4] = __builtin_bit_cast(uint32_t, e[j]);
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(S) / 2; ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
    }
    // a use of the words from here on converts them again, instead of keeping what was converted before
    __device__ __forceinline__ void again() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(S) / 2; ++i) asm("" : "+v"(w[i]));
    }
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (sizeof(S) == 2)
            return __builtin_bit_cast(float, j & 1 ? (uint32_t)w[0][j >> 1] & 0xFFFF0000u : (uint32_t)w[0][j >> 1] << 16);
        else
            return __builtin_bit_cast(float, (uint32_t)w[j / 4][j % 4]);
    }
};

struct NormArgs {
    int64_t tokens, ld;            // ld: row pitch of every [tokens][d] array
    int d, gate_kind;
    float scale, eps;
    const void* gate;              // fp32 [d] or bf16 [tokens][ld]
    const float *w_post, *w_pre;
};

// A row per WPR waves of CH chunks of 8 elements per lane, four rows per workgroup where a wave has one: the row stays in registers
// between its two sums, and thousands of rows in flight keep HBM busy.  4096 x 2048, fp32 stream, channel gate: 19.5 us (5.2 TB/s);
// 8192 x 4096, bf16: 53 us (5.1 TB/s); one token of 4096: 3.3 us, the latency of a load, two sums and a store.
template <typename S, int WPR, int CH>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void k_residual_norm_fwd(NormArgs a, const S* h, const uint16_t* __restrict__ y,
                                                                                S* h_out, uint16_t* __restrict__ u) {
    constexpr int NT = 64 * WPR, ROWS = WPR == 1 ? 4 : 1;
    __shared__ float slots[2][WPR];
    const int64_t t = (int64_t)blockIdx.x * ROWS + (WPR == 1 ? threadIdx.x >> 6 : 0);
    if (WPR == 1 && t >= a.tokens) return;
    const int tid = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t row = t * a.ld;
    float hv[CH][8], yv[CH][8];
    float ss[1] = {0.f};
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const int c = 8 * (tid + NT * q), valid = a.d - c;
        load8(h + row + c, valid, hv[q]);
        if (y != nullptr) load8(y + row + c, valid, yv[q]);
    }
    if (y != nullptr) {
        float inv = 1.f;
        if (a.w_post != nullptr) {
#pragma unroll
            for (int q = 0; q < CH; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) ss[0] = __builtin_fmaf(yv[q][j], yv[q][j], ss[0]);
            row_sums<1, WPR>(ss, slots[0]);
            inv = 1.f / sqrtf(ss[0] / (float)a.d + a.eps);
        }
        const float k = a.scale * inv;
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = 8 * (tid + NT * q), valid = a.d - c;
            float g[8];
            if (a.w_post != nullptr) {
                load8(a.w_post + c, valid, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) yv[q][j] *= g[j];
            }
            if (a.gate_kind != kGateNone) {
                if (a.gate_kind == kGateChannel) load8(static_cast<const float*>(a.gate) + c, valid, g);
                else load8(static_cast<const uint16_t*>(a.gate) + row + c, valid, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) yv[q][j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) hv[q][j] = __builtin_fmaf(k, yv[q][j], hv[q][j]);
            store8(h_out + row + c, valid, hv[q]);
        }
    }
    if (u == nullptr) return;
    ss[0] = 0.f;
#pragma unroll
    for (int q = 0; q < CH; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) ss[0] = __builtin_fmaf(hv[q][j], hv[q][j], ss[0]);
    row_sums<1, WPR>(ss, slots[1]);
    const float inv = 1.f / sqrtf(ss[0] / (float)a.d + a.eps);
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const int c = 8 * (tid + NT * q), valid = a.d - c;
        float g[8];
        load8(a.w_pre + c, valid, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = hv[q][j] * inv * g[j];
        store8(u + row + c, valid, g);
    }
}

// The sums over a row that dh and dy need are all known ahead of dh: mean(k dh y) is linear in dh = dh' + r a - r c h', so
// one reduction of six sums serves both norms.  A workgroup has ROWS rows at a time, `per` times, and keeps the columns' sums over
// them in registers: dw_pre's, and E = sum_t dh y q (times the gate where that is per token), of which dw_post and a channel's dgate
// are multiples.  At its end the ROWS sums are added in order.
// CH == 1 (rows of up to 8192): the vectors stay in registers; with two chunks per lane there are none left for them.  (Fetching the next
// rows ahead of the present ones' sums as well: 8192 x 4096 the same, 4096 x 2048 with a gate per token 65 us against 38, for the registers
// that it spills.)  Two chunks per lane and their columns' sums do not fit either: 116 to 190 registers of a lane live in scratch, and 8192
// x 16384, bf16, takes 831 us (1.9 TB/s), 4096 x 9216 371, where 4096 x 8192 takes 96 (4.2 TB/s).  8 elements per lane and 16 waves per
// workgroup instead of 16 and 4, which took twice the registers and twice the partial sums: 8192 x 4096, bf16, 112 us -> 88 (4.6 TB/s); 4096
// x 2048, fp32 stream, gate per token 38 us (4.8 TB/s); 1000 x 2047 of the same 16 us, one row per wave group: latency.
template <typename S, int WPR, int CH, int ROWS, bool TOKEN_GATE>
__global__ __launch_bounds__(64 * WPR * ROWS, 4) void k_residual_norm_bwd(
    NormArgs a, const uint16_t* __restrict__ du, const S* dh_next, const S* __restrict__ h, const uint16_t* __restrict__ y, S* dh,
    uint16_t* __restrict__ dy, uint16_t* __restrict__ dgate, float* __restrict__ part, int per) {
    constexpr int NT = 64 * WPR;
    constexpr bool kHold = CH == 1;
    __shared__ float slots[2][WPR * ROWS * 6];
    const int tid = threadIdx.x % NT, sub = __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    const bool post = a.w_post != nullptr, has_y = y != nullptr, has_u = du != nullptr;
    const float rd = 1.f / (float)a.d;
    float sum_pre[CH][8], sum_e[CH][8];
#pragma unroll
    for (int q = 0; q < CH; ++q)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum_pre[q][j] = sum_e[q][j] = 0.f;
    // wk: scale * w_post (* gate of the channel), wp: w_pre
    auto vectors = [&](int q, float (&wk)[8], float (&wp)[8]) {
        const int c = 8 * (tid + NT * q), valid = a.d - c;
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            wk[j] = a.scale;
            wp[j] = 0.f;
        }
        if (has_u) load8(a.w_pre + c, valid, wp);
        if (post) {
            load8(a.w_post + c, valid, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) wk[j] *= g[j];
        }
        if (a.gate_kind == kGateChannel) {
            load8(static_cast<const float*>(a.gate) + c, valid, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) wk[j] *= g[j];
        }
    };
    struct Row {
        Raw8<S> h[CH], d[CH];
        Raw8<uint16_t> u[CH], y[CH], g[TOKEN_GATE ? CH : 1];
    };
    auto fetch = [&](Row& w, int64_t t) {
        const int64_t row = t * a.ld;
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = 8 * (tid + NT * q), valid = t < a.tokens ? a.d - c : 0;   // past the end: zeros, which add nothing
            if (has_u) {
                w.h[q].load(h + row + c, valid);
                w.u[q].load(du + row + c, valid);
            } else {
                w.h[q].zero();
                w.u[q].zero();
            }
            if (dh_next != nullptr) w.d[q].load(dh_next + row + c, valid);
            else w.d[q].zero();
            if (has_y) w.y[q].load(y + row + c, valid);
            else w.y[q].zero();
            if constexpr (TOKEN_GATE) w.g[q].load(static_cast<const uint16_t*>(a.gate) + row + c, valid);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * per * ROWS + sub;
    Row w;
    fetch(w, first);                                       // ahead of the vectors: one latency for both
    float held_k[8], held_p[8];
    if constexpr (kHold) vectors(0, held_k, held_p);
    auto compute = [&](Row& w, int64_t t, float* slot) {
        const int64_t row = t * a.ld;
        float s[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};   // h h, a h, y y, k y dh', k y a, k y h
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            float wk[8], wp[8];
            if constexpr (!kHold) vectors(q, wk, wp);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float hh = w.h[q][j], av = w.u[q][j] * (kHold ? held_p[j] : wp[j]), yy = w.y[q][j];
                float ky = yy * (kHold ? held_k[j] : wk[j]);
                if constexpr (TOKEN_GATE) ky *= w.g[q][j];
                s[0] = __builtin_fmaf(hh, hh, s[0]);
                s[1] = __builtin_fmaf(av, hh, s[1]);
                s[2] = __builtin_fmaf(yy, yy, s[2]);
                s[3] = __builtin_fmaf(ky, w.d[q][j], s[3]);
                s[4] = __builtin_fmaf(ky, av, s[4]);
                s[5] = __builtin_fmaf(ky, hh, s[5]);
            }
        }
        row_sums<6, WPR>(s, slot);
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            w.h[q].again();
            w.d[q].again();
            w.u[q].again();
            w.y[q].again();
            if constexpr (TOKEN_GATE) w.g[q].again();
        }
        // (past the end: r = q = 0, so that zeros add nothing with eps = 0 either; r and q are multiplied into the sums one by one, since
        // the square of one overflows where eps is tiny and the row zero)
        const bool row_is = t < a.tokens;
        const float r = has_u && row_is ? 1.f / sqrtf(s[0] * rd + a.eps) : 0.f;
        const float qi = !post ? 1.f : row_is ? 1.f / sqrtf(s[2] * rd + a.eps) : 0.f;
        const float c1 = r * (r * s[1]) * rd;                                             // dh = dh' + r (a - c1 h')
        const float c2 = post ? qi * (qi * (s[3] + r * (s[4] - c1 * s[5]))) * rd : 0.f;   // dy = q (k dh - c2 y)
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = 8 * (tid + NT * q), valid = t < a.tokens ? a.d - c : 0;
            float wk[8], wp[8], o[8], p[8], e[8];
            if constexpr (!kHold) vectors(q, wk, wp);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float gt = 1.f;
                if constexpr (TOKEN_GATE) gt = w.g[q][j];
                const float uu = w.u[q][j], hh = w.h[q][j], yy = w.y[q][j], k = kHold ? held_k[j] : wk[j];
                sum_pre[q][j] = __builtin_fmaf(uu * hh, r, sum_pre[q][j]);
                o[j] = __builtin_fmaf(r, __builtin_fmaf(-c1, hh, uu * (kHold ? held_p[j] : wp[j])), w.d[q][j]);
                p[j] = qi * __builtin_fmaf(-c2, yy, k * gt * o[j]);
                const float x = o[j] * yy * qi;
                e[j] = k * x;
                sum_e[q][j] = __builtin_fmaf(x, gt, sum_e[q][j]);
            }
            store8(dh + row + c, valid, o);
            if (has_y) store8(dy + row + c, valid, p);
            if constexpr (TOKEN_GATE)
                if (dgate != nullptr) store8(dgate + row + c, valid, e);
        }
    };
    for (int i = 0; i < per; ++i) {
        const int64_t t = first + (int64_t)i * ROWS;
        compute(w, t, slots[i & 1]);
        if (i + 1 < per) fetch(w, t + ROWS);
    }
    if (part == nullptr) return;
    if constexpr (ROWS > 1) {
        __shared__ float sums[ROWS - 1][2 * 8 * CH * NT];
        if (sub != 0)
#pragma unroll
            for (int q = 0; q < CH; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sums[sub - 1][(q * 8 + j) * NT + tid] = sum_pre[q][j];
                    sums[sub - 1][((CH + q) * 8 + j) * NT + tid] = sum_e[q][j];
                }
        __syncthreads();
        if (sub != 0) return;
#pragma unroll
        for (int q = 0; q < CH; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 0; w < ROWS - 1; ++w) {
                    sum_pre[q][j] += sums[w][(q * 8 + j) * NT + tid];
                    sum_e[q][j] += sums[w][((CH + q) * 8 + j) * NT + tid];
                }
    }
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const int c = 8 * (tid + NT * q), valid = a.d - c;
        float* to = part + (int64_t)blockIdx.x * 2 * a.d + c;
        if (has_u) store8(to, valid, sum_pre[q]);
        if (has_y) store8(to + a.d, valid, sum_e[q]);
    }
}

// Columns' sums over the workgroups' partial ones, in a fixed order: 32 of the 2 d columns per workgroup, 32 slices of the groups.  4 to
// 5 us at 250 groups (64 columns and 16 slices: 10 us at 512), mostly latency.
__global__ __launch_bounds__(1024) void k_residual_norm_cols(NormArgs a, const float* __restrict__ part, int groups, bool has_u, bool has_y,
                                                             float* __restrict__ dw_pre, float* __restrict__ dw_post,
                                                             float* __restrict__ dgate) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;                       // below d: dw_pre's, then E's
    const bool mine = col < 2 * a.d && (col < a.d ? has_u : has_y);
    float s = 0.f;
    if (mine) {
        const float* p = part + col;
        const int64_t step = (int64_t)32 * 2 * a.d;
        p += (int64_t)slice * 2 * a.d;
#pragma unroll 8
        for (int g = slice; g < groups; g += 32, p += step) s += *p;
    }
    sums[slice][lane] = s;
    __syncthreads();
    if (slice != 0 || !mine) return;
#pragma unroll
    for (int w = 1; w < 32; ++w) s += sums[w][lane];
    if (col < a.d) {
        if (dw_pre != nullptr) dw_pre[col] = s;
    } else {
        const int j = col - a.d;
        s *= a.scale;
        const float g = a.gate_kind == kGateChannel ? static_cast<const float*>(a.gate)[j] : 1.f;
        if (dw_post != nullptr) dw_post[j] = s * g;
        if (dgate != nullptr) dgate[j] = s * (a.w_post != nullptr ? a.w_post[j] : 1.f);
    }
}

// Rows of d elements: up to 1024 a wave, up to 4096 four waves, then 8 and 16.  f(waves per row, chunks per lane).
template <typename F>
static void norm_shape(int64_t d, F f) {
    using std::integral_constant;
    if (d <= 512) f(integral_constant<int, 1>(), integral_constant<int, 1>());
    else if (d <= 1024) f(integral_constant<int, 1>(), integral_constant<int, 2>());
    else if (d <= 2048) f(integral_constant<int, 4>(), integral_constant<int, 1>());
    else if (d <= 4096) f(integral_constant<int, 4>(), integral_constant<int, 2>());
    else if (d <= 8192) f(integral_constant<int, 8>(), integral_constant<int, 2>());
    else f(integral_constant<int, 16>(), integral_constant<int, 2>());
}
// ... of the backward pass: f(waves per row, chunks per lane, rows per workgroup).
template <typename F>
static void norm_bwd_shape(int64_t d, F f) {
    using std::integral_constant;
    if (d <= 512) f(integral_constant<int, 1>(), integral_constant<int, 1>(), integral_constant<int, 8>());
    else if (d <= 1024) f(integral_constant<int, 2>(), integral_constant<int, 1>(), integral_constant<int, 4>());
    else if (d <= 2048) f(integral_constant<int, 4>(), integral_constant<int, 1>(), integral_constant<int, 4>());
    else if (d <= 4096) f(integral_constant<int, 8>(), integral_constant<int, 1>(), integral_constant<int, 2>());
    else if (d <= 8192) f(integral_constant<int, 16>(), integral_constant<int, 1>(), integral_constant<int, 1>());
    else f(integral_constant<int, 16>(), integral_constant<int, 2>(), integral_constant<int, 1>());
}

// Workgroups of the backward pass and the rows that they take in turn.
struct NormSplit {
    int per, groups;
};
static NormSplit norm_split(int64_t tokens, int64_t d) {
    int64_t rows = 1;
    norm_bwd_shape(d, [&](auto, auto, auto r) { rows = r.value; });
    const int64_t most = 256;
    const int64_t per = (tokens + rows * most - 1) / (rows * most);
    return {(int)per, (int)((tokens + rows * per - 1) / (rows * per))};
}

static int check_norm(int64_t tokens, int64_t d, int64_t& ld) {
    if (tokens <= 0 || d <= 0 || d > kNormMaxD || tokens >= kNormMaxTokens) return QG_ERR_SHAPE;
    if (ld == 0) ld = d;
    if (ld != d && (ld < d || (ld & 15))) return QG_ERR_SHAPE;
    if (ld >= (int64_t(1) << 31)) return QG_ERR_SHAPE;
    return QG_OK;
}

}  // namespace qg

using namespace qg;

extern "C" int qg_residual_norm_forward(const void* h, const uint16_t* y_bf16, const float* w_post, const void* gate, int gate_kind,
                                        const float* w_pre, float scale, float eps, int64_t tokens, int64_t d, int64_t ld,
                                        int stream_fp32, void* h_out, uint16_t* u_bf16, void* stream) {
    if (!h || (!y_bf16 && !u_bf16) || (y_bf16 && !h_out) || (u_bf16 && !w_pre)) return QG_ERR_NULL;
    if (gate_kind < QG_GATE_NONE || gate_kind > QG_GATE_TOKEN) return QG_ERR_SHAPE;
    if (y_bf16 && gate_kind != QG_GATE_NONE && !gate) return QG_ERR_NULL;
    if (int e = check_norm(tokens, d, ld)) return e;
    for (const void* p : {h, (const void*)y_bf16, (const void*)w_post, gate, (const void*)w_pre, (const void*)h_out, (const void*)u_bf16})
        if (!aligned16(p)) return QG_ERR_ALIGN;
    const NormArgs a = {tokens, ld, (int)d, gate_kind, scale, eps, gate, w_post, w_pre};
    norm_shape(d, [&](auto wpr, auto ch) {
        const unsigned grid = (unsigned)(wpr.value == 1 ? (tokens + 3) / 4 : tokens);
        const dim3 block(wpr.value == 1 ? 256 : 64 * wpr.value);
        if (stream_fp32)
            hipLaunchKernelGGL((k_residual_norm_fwd<float, wpr.value, ch.value>), dim3(grid), block, 0, (hipStream_t)stream, a,
                               static_cast<const float*>(h), y_bf16, static_cast<float*>(h_out), u_bf16);
        else
            hipLaunchKernelGGL((k_residual_norm_fwd<uint16_t, wpr.value, ch.value>), dim3(grid), block, 0, (hipStream_t)stream, a,
                               static_cast<const uint16_t*>(h), y_bf16, static_cast<uint16_t*>(h_out), u_bf16);
    });
    return check_launch();
}

extern "C" size_t qg_residual_norm_workspace_bytes(int64_t tokens, int64_t d) {
    int64_t ld = 0;
    if (check_norm(tokens, d, ld)) return 0;
    return (size_t)norm_split(tokens, d).groups * 2 * (size_t)d * 4;
}

extern "C" int qg_residual_norm_backward(const uint16_t* du_bf16, const void* dh_next, const void* h_next, const uint16_t* y_bf16,
                                         const float* w_post, const void* gate, int gate_kind, const float* w_pre, float scale,
                                         float eps, int64_t tokens, int64_t d, int64_t ld, int stream_fp32, void* dh,
                                         uint16_t* dy_bf16, float* dw_pre, float* dw_post, void* dgate, void* workspace,
                                         size_t workspace_bytes, void* stream) {
    if ((!du_bf16 && !dh_next) || !dh || (du_bf16 && (!h_next || !w_pre)) || (y_bf16 && !dy_bf16)) return QG_ERR_NULL;
    if ((dw_pre && !du_bf16) || (dw_post && (!y_bf16 || !w_post))) return QG_ERR_NULL;
    if (gate_kind < QG_GATE_NONE || gate_kind > QG_GATE_TOKEN) return QG_ERR_SHAPE;
    if (y_bf16 && gate_kind != QG_GATE_NONE && !gate) return QG_ERR_NULL;
    if (dgate && (!y_bf16 || gate_kind == QG_GATE_NONE)) return QG_ERR_NULL;
    if (int e = check_norm(tokens, d, ld)) return e;
    for (const void* p : {(const void*)du_bf16, dh_next, h_next, (const void*)y_bf16, (const void*)w_post, gate, (const void*)w_pre,
                          (const void*)dh, (const void*)dy_bf16, (const void*)dw_pre, (const void*)dw_post, (const void*)dgate,
                          (const void*)workspace})
        if (!aligned16(p)) return QG_ERR_ALIGN;
    const bool dgate_cols = dgate != nullptr && gate_kind == QG_GATE_CHANNEL, cols = dw_pre || dw_post || dgate_cols;
    if (cols && (!workspace || workspace_bytes < qg_residual_norm_workspace_bytes(tokens, d))) return QG_ERR_WORKSPACE;
    if (!y_bf16) gate_kind = QG_GATE_NONE;
    const NormArgs a = {tokens, ld, (int)d, gate_kind, scale, eps, gate, y_bf16 ? w_post : nullptr, w_pre};
    const NormSplit split = norm_split(tokens, d);
    float* part = cols ? static_cast<float*>(workspace) : nullptr;
    uint16_t* dgate_tokens = gate_kind == QG_GATE_TOKEN ? static_cast<uint16_t*>(dgate) : nullptr;
    norm_bwd_shape(d, [&](auto wpr, auto ch, auto rows) {
        auto launch = [&](auto s, auto token) {
            using S = decltype(s);
            hipLaunchKernelGGL((k_residual_norm_bwd<S, wpr.value, ch.value, rows.value, token.value>), dim3((unsigned)split.groups),
                               dim3(64 * wpr.value * rows.value), 0, (hipStream_t)stream, a, du_bf16, static_cast<const S*>(dh_next),
                               static_cast<const S*>(h_next), y_bf16, static_cast<S*>(dh), dy_bf16, dgate_tokens, part, split.per);
        };
        auto pick = [&](auto s) { gate_kind == QG_GATE_TOKEN ? launch(s, std::true_type()) : launch(s, std::false_type()); };
        stream_fp32 ? pick(float()) : pick(uint16_t());
    });
    if (cols)
        hipLaunchKernelGGL(k_residual_norm_cols, dim3((unsigned)((2 * d + 31) / 32)), dim3(1024), 0, (hipStream_t)stream, a, part,
                           split.groups, du_bf16 != nullptr, y_bf16 != nullptr, dw_pre, dw_post,
                           dgate_cols ? static_cast<float*>(dgate) : nullptr);
    return check_launch();
}
