// The INT8 linear layer with an epilogue (bias, activation, residual), and the gated pair of layers that opens a decoder's
// feed-forward block, with their backward passes.
//     act forward:     z = x W^T + bias,  y = act(z) + residual
//     act backward:    dz = dy act'(z),   dx = dz W,  G = dz^T x,  dbias = sum over tokens of dz
//     gated forward:   y = act(x Wg^T) * (x Wu^T)
//     gated backward:  dzg = dy zu act'(zg),  dzu = dy act(zg),  dx = dzg Wg + dzu Wu,  Gg = dzg^T x,  Gu = dzu^T x
// W is dequantized while it is staged, as in the plain layer.  The forward passes are one launch: the activation is applied to
// the fp32 sums, and z is rounded only where it is stored for the backward pass.  dz goes through memory as bf16 (it is an
// operand of two products), made by one pass over dy and z.
#include "qg_epilogue.h"

namespace qg {

static int check_sizes(int64_t tokens, int64_t m, int64_t n, int group) {
    const int64_t lim = int64_t(1) << 31;
    if (tokens <= 0 || m <= 0 || n <= 0 || tokens >= lim / m || tokens >= lim / n || m >= lim / n) return QG_ERR_SHAPE;
    if (group != kGroup) return QG_ERR_GROUP;
    return QG_OK;
}
static int check_pitch(int64_t rows, int64_t len, int64_t& ld) {
    if (ld == 0) ld = len;
    if (ld != len && (ld < len || (ld & 15))) return QG_ERR_SHAPE;
    if (rows >= (int64_t(1) << 31) / ld) return QG_ERR_SHAPE;
    return QG_OK;
}
static bool all_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned16(p)) return false;
    return true;
}

// ---- dz: 8 columns of a row per thread, 512 columns and every 4th row of a slab per wave.  Bound by HBM (6 bytes per element, a
// pair 10).  dbias: the columns' sums over a slab from registers, the four waves added in order, slabs added by k_column_sums.
template <bool PAIR>
__global__ __launch_bounds__(256) void k_act_backward(const uint16_t* dy, const uint16_t* zg, const uint16_t* zu, uint16_t* dzg,
                                                      uint16_t* dzu, float* __restrict__ part, int tokens, int m, int64_t ld, int rows,
                                                      int kind) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * 512 + lane * 8, left = m - col;
    const int first = blockIdx.y * rows, last = min(first + rows, tokens);
    float sum[8] = {};
    if (left > 0) {
        for (int t = first + wave; t < last; t += 4) {
            const int64_t at = (int64_t)t * ld + col;
            float d[8], z[8], o[8];
            load_run(dy + at, left, d);
            if constexpr (PAIR) {
                float u[8], p[8];
                load_run(zg + at, left, z);
                load_run(zu + at, left, u);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float a;
                    const float g = act_grad(z[e], kind, a);
                    o[e] = d[e] * u[e] * g;
                    p[e] = d[e] * a;
                }
                store_run(dzg + at, left, o);
                store_run(dzu + at, left, p);
            } else {
                if (kind != QG_ACT_NONE) {
                    load_run(zg + at, left, z);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float a;
                        o[e] = d[e] * act_grad(z[e], kind, a);
                    }
                    if (dzg != nullptr) store_run(dzg + at, left, o);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = d[e];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += o[e];
            }
        }
    }
    if (PAIR || part == nullptr) return;
    __shared__ float sums[4][512];
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][e * 64 + lane] = sum[e];
    __syncthreads();
    if (wave != 0 || left <= 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int w = 1; w < 4; ++w) sum[e] += sums[w][e * 64 + lane];
        if (e < left) part[(int64_t)blockIdx.y * m + col + e] = sum[e];
    }
}

// out[j] = sum over the slabs of part[slab][j], in a fixed order: 64 columns per workgroup, 16 waves.
__global__ __launch_bounds__(1024) void k_column_sums(const float* __restrict__ part, int slabs, int m, float* __restrict__ out) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (col < m)
        for (int g = wave; g < slabs; g += 16) s += part[(int64_t)g * m + col];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= m) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    out[col] = s;
}

// Rows of a slab, and slabs: about a thousand workgroups where there are rows for them.
struct Slabs {
    int rows, count;
};
static Slabs act_slabs(int64_t tokens, int64_t m) {
    const int64_t across = (m + 511) / 512, want = (1024 + across - 1) / across;
    int64_t rows = (tokens + want - 1) / want;
    rows = (rows + 3) / 4 * 4;
    return {(int)rows, (int)((tokens + rows - 1) / rows)};
}

template <bool PAIR>
static int launch_act_backward(const uint16_t* dy, const uint16_t* zg, const uint16_t* zu, uint16_t* dzg, uint16_t* dzu, float* part,
                               int64_t tokens, int64_t m, int64_t ld, int kind, hipStream_t st) {
    const Slabs s = act_slabs(tokens, m);
    hipLaunchKernelGGL((k_act_backward<PAIR>), dim3((unsigned)((m + 511) / 512), (unsigned)s.count), dim3(256), 0, st, dy, zg, zu, dzg, dzu,
                       part, (int)tokens, (int)m, ld, s.rows, kind);
    return check_launch();
}

// Tiles of the products with an epilogue, x W^T of one weight.
template <typename EPI>
static int launch_act_forward(EpiProduct<LinOperand, EPI> p, hipStream_t st) {
    const int64_t t32 = (int64_t)((p.M + 31) / 32) * ((p.N + 31) / 32), t128 = (int64_t)((p.M + 127) / 128) * ((p.N + 127) / 128);
    if (t32 <= 256) return launch_epilogue_ksplit<kBf16KFast, kInt8KFast, 8, 1>(p, st);
    if (t32 <= 768) return launch_epilogue_ksplit<kBf16KFast, kInt8KFast, 4, 1>(p, st);
    if (p.M >= 1024 && (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256) >= 256)
        return launch_epilogue_shape<kBf16KFast, kInt8KFast, 2, 256, 64, 4, true, true, 1, 1>(p, st);
    if (t128 < 256) return launch_epilogue_shape<kBf16KFast, kInt8KFast, 1, 64, 64, 2, true, true, 1, 1>(p, st);
    return launch_epilogue_shape<kBf16KFast, kInt8KFast, 2, 128, 64, 2, true, true, 1, 1>(p, st);
}

// ... of a pair: N columns of each.
template <typename EPI>
static int launch_gated_forward(EpiProduct<LinPairOperand, EPI> p, hipStream_t st) {
    const int64_t t32 = (int64_t)((p.M + 31) / 32) * ((p.N + 31) / 32);
    if (t32 <= 256) return launch_epilogue_ksplit<kBf16KFast, kInt8KFast, 8, 1>(p, st);
    if (t32 <= 768) return launch_epilogue_ksplit<kBf16KFast, kInt8KFast, 4, 1>(p, st);
    if (p.M >= 1024 && (int64_t)((p.M + 255) / 256) * ((p.N + 127) / 128) >= 256)
        return launch_epilogue_shape<kBf16KFast, kInt8KFast, 2, 256, 64, 4, true, true, 1, 1>(p, st);
    return launch_epilogue_shape<kBf16KFast, kInt8KFast, 2, 128, 64, 2, true, true, 1, 1>(p, st);
}

// dx = dzg Wg + dzu Wu
static int launch_gated_dx(EpiProduct<LinOperand, PlainEpilogue<uint16_t>> p, hipStream_t st) {
    const int64_t t32 = (int64_t)((p.M + 31) / 32) * ((p.N + 31) / 32), t128 = (int64_t)((p.M + 127) / 128) * ((p.N + 127) / 128);
    if (t32 <= 512) return launch_epilogue_ksplit<kBf16KFast, kInt8KSlow, 4, 2>(p, st);
    if (p.M >= 1024 && (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256) >= 256)
        return launch_epilogue_shape<kBf16KFast, kInt8KSlow, 2, 256, 64, 4, true, true, 1, 2>(p, st);
    if (t128 < 160) return launch_epilogue_shape<kBf16KFast, kInt8KSlow, 1, 64, 64, 2, true, true, 1, 2>(p, st);
    return launch_epilogue_shape<kBf16KFast, kInt8KSlow, 2, 128, 64, 2, true, true, 1, 2>(p, st);
}

}  // namespace qg

using namespace qg;

extern "C" int qg_int8_linear_act_forward(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const uint16_t* bias_bf16,
                                          const uint16_t* residual_bf16, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n,
                                          int64_t ld_m, int group, uint16_t* z_bf16, uint16_t* y_bf16, void* stream) {
    if (!x_bf16 || !Wq || !Ws || !y_bf16) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_sizes(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({x_bf16, Wq, Ws, bias_bf16, residual_bf16, z_bf16, y_bf16})) return QG_ERR_ALIGN;
    EpiProduct<LinOperand, RunEpilogue<ActRun>> p;
    p.A = p.A2 = LinOperand{x_bf16, nullptr, ld_n, 0};
    p.B = p.B2 = LinOperand{Wq, Ws, ld_n, (int)((n + kGroup - 1) / kGroup)};
    static_cast<ActRun&>(p.epi) = ActRun{bias_bf16, residual_bf16, z_bf16, y_bf16, ld_m, act};
    p.M = (int)tokens, p.N = (int)m, p.K = (int)n;
    return launch_act_forward(p, (hipStream_t)stream);
}

extern "C" size_t qg_int8_linear_act_workspace_bytes(int64_t tokens, int64_t m) {
    if (tokens <= 0 || m <= 0 || tokens >= (int64_t(1) << 31) / m) return 0;
    return (size_t)act_slabs(tokens, m).count * (size_t)m * 4;
}

extern "C" int qg_int8_linear_act_backward(const uint16_t* dy_bf16, const uint16_t* z_bf16, const uint16_t* x_bf16, const int8_t* Wq,
                                           const float* Ws, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m,
                                           int group, uint16_t* dz_bf16, uint16_t* dx_bf16, uint16_t* G_bf16, float* dbias,
                                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy_bf16 || (!dx_bf16 && !G_bf16 && !dbias)) return QG_ERR_NULL;
    if ((dx_bf16 && (!Wq || !Ws)) || (G_bf16 && !x_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    const bool products = dx_bf16 || G_bf16;
    if (act != QG_ACT_NONE && (!z_bf16 || (products && !dz_bf16))) return QG_ERR_NULL;
    if (int e = check_sizes(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({dy_bf16, z_bf16, x_bf16, Wq, Ws, dz_bf16, dx_bf16, G_bf16, dbias, workspace})) return QG_ERR_ALIGN;
    if (dbias && (!workspace || workspace_bytes < qg_int8_linear_act_workspace_bytes(tokens, m))) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    float* part = dbias ? static_cast<float*>(workspace) : nullptr;
    const uint16_t* dz = dy_bf16;
    if (act != QG_ACT_NONE || dbias) {
        uint16_t* out = act != QG_ACT_NONE && products ? dz_bf16 : nullptr;
        if (int e = launch_act_backward<false>(dy_bf16, z_bf16, nullptr, out, nullptr, part, tokens, m, ld_m, act, st)) return e;
        if (out) dz = out;
    }
    if (dbias) {
        hipLaunchKernelGGL(k_column_sums, dim3((unsigned)((m + 63) / 64)), dim3(1024), 0, st, part, act_slabs(tokens, m).count, (int)m, dbias);
        if (int e = check_launch()) return e;
    }
    if (!products) return QG_OK;
    return qg_int8_linear_backward_ld(dz, x_bf16, Wq, Ws, tokens, m, n, ld_n, ld_m, group, dx_bf16, G_bf16, stream);
}

extern "C" int qg_int8_gated_forward(const uint16_t* x_bf16, const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus,
                                     int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group,
                                     uint16_t* zg_bf16, uint16_t* zu_bf16, uint16_t* y_bf16, void* stream) {
    if (!x_bf16 || !Wgq || !Wgs || !Wuq || !Wus || !y_bf16 || (!zg_bf16 != !zu_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_sizes(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({x_bf16, Wgq, Wgs, Wuq, Wus, zg_bf16, zu_bf16, y_bf16})) return QG_ERR_ALIGN;
    EpiProduct<LinPairOperand, RunEpilogue<GatedRun>> p;
    p.A = p.A2 = LinOperand{x_bf16, nullptr, ld_n, 0};
    static_cast<LinOperand&>(p.B) = LinOperand{Wgq, Wgs, ld_n, (int)((n + kGroup - 1) / kGroup)};
    p.B.base2 = Wuq;
    p.B.scales2 = Wus;
    p.B2 = p.B;
    static_cast<GatedRun&>(p.epi) = GatedRun{zg_bf16, zu_bf16, y_bf16, ld_m, act};
    p.M = (int)tokens, p.N = (int)m, p.K = (int)n;
    return launch_gated_forward(p, (hipStream_t)stream);
}

extern "C" int qg_int8_gated_backward(const uint16_t* dy_bf16, const uint16_t* zg_bf16, const uint16_t* zu_bf16, const uint16_t* x_bf16,
                                      const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus, int act, int64_t tokens,
                                      int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group, uint16_t* dzg_bf16, uint16_t* dzu_bf16,
                                      uint16_t* dx_bf16, uint16_t* Gg_bf16, uint16_t* Gu_bf16, void* stream) {
    if (!dy_bf16 || !zg_bf16 || !zu_bf16 || !dzg_bf16 || !dzu_bf16 || (!Gg_bf16 != !Gu_bf16) || (!dx_bf16 && !Gg_bf16)) return QG_ERR_NULL;
    if ((dx_bf16 && (!Wgq || !Wgs || !Wuq || !Wus)) || (Gg_bf16 && !x_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_sizes(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({dy_bf16, zg_bf16, zu_bf16, x_bf16, Wgq, Wgs, Wuq, Wus, dzg_bf16, dzu_bf16, dx_bf16, Gg_bf16, Gu_bf16}))
        return QG_ERR_ALIGN;
    const hipStream_t st = (hipStream_t)stream;
    if (int e = launch_act_backward<true>(dy_bf16, zg_bf16, zu_bf16, dzg_bf16, dzu_bf16, nullptr, tokens, m, ld_m, act, st)) return e;
    const int sg = (int)((n + kGroup - 1) / kGroup);
    const LinOperand dzg = {dzg_bf16, nullptr, ld_m, 0}, dzu = {dzu_bf16, nullptr, ld_m, 0};
    if (dx_bf16) {
        EpiProduct<LinOperand, PlainEpilogue<uint16_t>> p;
        p.A = dzg, p.A2 = dzu;
        p.B = LinOperand{Wgq, Wgs, ld_n, sg}, p.B2 = LinOperand{Wuq, Wus, ld_n, sg};
        p.epi = PlainEpilogue<uint16_t>{nullptr, dx_bf16, ld_n};
        p.M = (int)tokens, p.N = (int)n, p.K = (int)m;
        if (int e = launch_gated_dx(p, st)) return e;
    }
    if (!Gg_bf16) return QG_OK;
    if (int e = qg_int8_linear_backward_ld(dzg_bf16, x_bf16, nullptr, nullptr, tokens, m, n, ld_n, ld_m, group, nullptr, Gg_bf16, stream))
        return e;
    return qg_int8_linear_backward_ld(dzu_bf16, x_bf16, nullptr, nullptr, tokens, m, n, ld_n, ld_m, group, nullptr, Gu_bf16, stream);
}
