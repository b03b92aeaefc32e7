// Norms of the residual stream: what stands between two blocks of a decoder, in one pass over the stream.  For every token
//     n  = w_post * y / rms(y)                    the norm behind a block (optional), y the block's output
//     h' = h + scale * gate * n                   its gate (none, one per channel, or one per token and channel), and the sum
//     u  = w_pre * h' / rms(h')                   the norm ahead of the next block (optional);  rms(v) = sqrt(mean v^2 + eps)
// and the gradients: with r = 1/rms(h'), q = 1/rms(y), a = w_pre du, k = scale * gate * w_post,
//     dh = dh' + r (a - h' r^2 mean(a h'))        of h and h' alike
//     dy = q (k dh - y q^2 mean(k dh y))
//     dw_pre = sum_t du h' r,   dw_post = sum_t scale gate dh y q,   dgate = scale dh w_post y q (summed over t if per channel)
// Every array is read or written once; a row stays in the registers of one workgroup (or wave).  All of it is bound by HBM.
#include "qg_common.h"
#include "qg_gemm_kernels.h"

namespace qg {

constexpr int kNormMaxD = 16384;
constexpr int64_t kNormMaxTokens = int64_t(1) << 22;   // (a workgroup of up to 1024 threads per token, 2^32 threads per launch)
enum : int { kGateNone = QG_GATE_NONE, kGateChannel = QG_GATE_CHANNEL, kGateToken = QG_GATE_TOKEN };

// 8 consecutive elements of a row, of which the first `valid` exist (the others read as 0); rows may start at any element.
__device__ __forceinline__ void load8(const uint16_t* p, int valid, float (&v)[8]) {
    u32x4 w = {0u, 0u, 0u, 0u};
    if (valid >= 8) {
        w = *reinterpret_cast<const u32x4_align2*>(p);
    } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < valid) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
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
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < valid ? p[j] : 0.f;
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

// Sums of N values over the WPR waves that share a row, the same value in every lane; `slot`: WPR * N floats of LDS, a set of
// its own for each of two calls in a row.  A fixed order: the result does not depend on timing.
template <int N, int WPR>
__device__ __forceinline__ void row_sums(float (&s)[N], float* slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_sum(s[i]);
    if constexpr (WPR > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) slot[wave * N + i] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t = slot[i];
#pragma unroll
            for (int w = 1; w < WPR; ++w) t += slot[w * N + i];
            s[i] = t;
        }
    }
}

struct NormArgs {
    int64_t tokens, ld;            // ld: row pitch of every [tokens][d] array
    int d, gate_kind;
    float scale, eps;
    const void* gate;              // fp32 [d] or bf16 [tokens][ld]
    const float *w_post, *w_pre;
};

// A row per WPR waves of CH chunks of 8 elements per lane; 4 / WPR rows per workgroup where a wave does.
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
// one reduction of six sums serves both norms.  A workgroup goes over `per` rows and keeps the columns' sums over them in
// registers: dw_pre's, and E = sum_t dh y q (times the gate where that is per token), of which dw_post and a channel's dgate
// are multiples.
template <typename S, int WPR, int CH>
__global__ __launch_bounds__(WPR == 1 ? 256 : 64 * WPR) void k_residual_norm_bwd(
    NormArgs a, const uint16_t* __restrict__ du, const S* dh_next, const S* __restrict__ h, const uint16_t* __restrict__ y, S* dh,
    uint16_t* __restrict__ dy, uint16_t* __restrict__ dgate, float* __restrict__ part, int64_t per) {
    constexpr int NT = 64 * WPR, WAVES = WPR == 1 ? 4 : WPR;
    __shared__ float slots[2][WPR * 6];
    const int tid = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
    const bool post = a.w_post != nullptr, has_y = y != nullptr, has_u = du != nullptr;
    const float rd = 1.f / (float)a.d;
    float sum_pre[CH][8], sum_e[CH][8], wk[CH][8], wp[CH][8];   // wk: scale * w_post (* gate of the channel)
#pragma unroll
    for (int q = 0; q < CH; ++q) {
        const int c = 8 * (tid + NT * q), valid = a.d - c;
        float g[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum_pre[q][j] = sum_e[q][j] = 0.f;
            wk[q][j] = a.scale;
            wp[q][j] = 0.f;
        }
        if (has_u) load8(a.w_pre + c, valid, wp[q]);
        if (post) {
            load8(a.w_post + c, valid, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) wk[q][j] *= g[j];
        }
        if (a.gate_kind == kGateChannel) {
            load8(static_cast<const float*>(a.gate) + c, valid, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) wk[q][j] *= g[j];
        }
    }
    const int64_t first = ((int64_t)blockIdx.x * (WPR == 1 ? 4 : 1) + (WPR == 1 ? threadIdx.x >> 6 : 0)) * per;
    const int64_t last = min(first + per, a.tokens);
    for (int64_t t = first; t < last; ++t) {
        const int64_t row = t * a.ld;
        float hv[CH][8], uv[CH][8], dv[CH][8], yv[CH][8], gv[CH][8];
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = 8 * (tid + NT * q), valid = a.d - c;
#pragma unroll
            for (int j = 0; j < 8; ++j) hv[q][j] = uv[q][j] = dv[q][j] = yv[q][j] = 0.f;
            if (has_u) {
                load8(h + row + c, valid, hv[q]);
                load8(du + row + c, valid, uv[q]);
            }
            if (dh_next != nullptr) load8(dh_next + row + c, valid, dv[q]);
            if (has_y) load8(y + row + c, valid, yv[q]);
            if (a.gate_kind == kGateToken) load8(static_cast<const uint16_t*>(a.gate) + row + c, valid, gv[q]);
        }
        float s[6] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};   // h h, a h, y y, k y dh', k y a, k y h
#pragma unroll
        for (int q = 0; q < CH; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float hh = hv[q][j], av = uv[q][j] * wp[q][j], yy = yv[q][j];
                const float ky = yy * wk[q][j] * (a.gate_kind == kGateToken ? gv[q][j] : 1.f);
                s[0] = __builtin_fmaf(hh, hh, s[0]);
                s[1] = __builtin_fmaf(av, hh, s[1]);
                s[2] = __builtin_fmaf(yy, yy, s[2]);
                s[3] = __builtin_fmaf(ky, dv[q][j], s[3]);
                s[4] = __builtin_fmaf(ky, av, s[4]);
                s[5] = __builtin_fmaf(ky, hh, s[5]);
            }
        row_sums<6, WPR>(s, slots[t & 1]);
        const float r = has_u ? 1.f / sqrtf(s[0] * rd + a.eps) : 0.f, qi = post ? 1.f / sqrtf(s[2] * rd + a.eps) : 1.f;
        const float c1 = r * r * s[1] * rd;                                        // dh = dh' + r (a - c1 h')
        const float c2 = post ? qi * qi * rd * (s[3] + r * (s[4] - c1 * s[5])) : 0.f;   // dy = q (k dh - c2 y)
#pragma unroll
        for (int q = 0; q < CH; ++q) {
            const int c = 8 * (tid + NT * q), valid = a.d - c;
            float o[8], p[8], e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gt = a.gate_kind == kGateToken ? gv[q][j] : 1.f;
                sum_pre[q][j] = __builtin_fmaf(uv[q][j] * hv[q][j], r, sum_pre[q][j]);
                o[j] = __builtin_fmaf(r, __builtin_fmaf(-c1, hv[q][j], uv[q][j] * wp[q][j]), dv[q][j]);
                p[j] = qi * __builtin_fmaf(-c2, yv[q][j], wk[q][j] * gt * o[j]);
                const float x = o[j] * yv[q][j] * qi;
                e[j] = wk[q][j] * x;
                sum_e[q][j] = __builtin_fmaf(x, gt, sum_e[q][j]);
            }
            store8(dh + row + c, valid, o);
            if (has_y) store8(dy + row + c, valid, p);
            if (dgate != nullptr) store8(dgate + row + c, valid, e);
        }
    }
    if (part == nullptr) return;
    if constexpr (WPR == 1) {   // the workgroup's four waves: their columns' sums through LDS, added in order
        __shared__ float sums[WAVES][2 * 512 * CH];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < CH; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[wave][(q * 8 + j) * 64 + tid] = sum_pre[q][j];
                sums[wave][((CH + q) * 8 + j) * 64 + tid] = sum_e[q][j];
            }
        __syncthreads();
        if (wave != 0) return;
#pragma unroll
        for (int q = 0; q < CH; ++q)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int w = 1; w < 4; ++w) {
                    sum_pre[q][j] += sums[w][(q * 8 + j) * 64 + tid];
                    sum_e[q][j] += sums[w][((CH + q) * 8 + j) * 64 + tid];
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

// Columns' sums over the workgroups' partial ones, in a fixed order: 64 columns of a row of 2 d per workgroup, 16 waves.
__global__ __launch_bounds__(1024) void k_residual_norm_cols(NormArgs a, const float* __restrict__ part, int groups, bool has_u, bool has_y,
                                                             float* __restrict__ dw_pre, float* __restrict__ dw_post,
                                                             float* __restrict__ dgate) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;                       // below d: dw_pre's, then E's
    const bool mine = col < 2 * a.d && (col < a.d ? has_u : has_y);
    float s = 0.f;
    if (mine)
        for (int g = wave; g < groups; g += 16) s += part[(int64_t)g * 2 * a.d + col];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || !mine) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
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

// Workgroups of the backward pass and the rows that a row's waves take in turn.
struct NormSplit {
    int64_t per;
    int groups;
};
static NormSplit norm_split(int64_t tokens, int64_t d) {
    const int64_t rows = d <= 1024 ? 4 : 1, most = 512;
    const int64_t per = (tokens + rows * most - 1) / (rows * most);
    return {per, (int)((tokens + rows * per - 1) / (rows * per))};
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
    norm_shape(d, [&](auto wpr, auto ch) {
        const dim3 grid((unsigned)split.groups), block(wpr.value == 1 ? 256 : 64 * wpr.value);
        if (stream_fp32)
            hipLaunchKernelGGL((k_residual_norm_bwd<float, wpr.value, ch.value>), grid, block, 0, (hipStream_t)stream, a, du_bf16,
                               static_cast<const float*>(dh_next), static_cast<const float*>(h_next), y_bf16, static_cast<float*>(dh),
                               dy_bf16, dgate_tokens, part, split.per);
        else
            hipLaunchKernelGGL((k_residual_norm_bwd<uint16_t, wpr.value, ch.value>), grid, block, 0, (hipStream_t)stream, a, du_bf16,
                               static_cast<const uint16_t*>(dh_next), static_cast<const uint16_t*>(h_next), y_bf16,
                               static_cast<uint16_t*>(dh), dy_bf16, dgate_tokens, part, split.per);
    });
    if (cols)
        hipLaunchKernelGGL(k_residual_norm_cols, dim3((unsigned)((2 * d + 63) / 64)), dim3(1024), 0, (hipStream_t)stream, a, part,
                           split.groups, du_bf16 != nullptr, y_bf16 != nullptr, dw_pre, dw_post,
                           dgate_cols ? static_cast<float*>(dgate) : nullptr);
    return check_launch();
}
