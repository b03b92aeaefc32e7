// The tile GEMM of qg_tile_gemm.h with work in its epilogue, while the sums are in registers and on their way through LDS: what
// the layers around the INT8 linear layer and the loss of a head are made of.
#pragma once
#include "qg_tile_gemm.h"

namespace qg {

// R consecutive bf16 elements (R: 4 or 8), of which the first `left` exist; the others read as 0.  (At a row's end the last element is
// read again in the place of those: loads that do not wait for each other.)
template <int R>
__device__ __forceinline__ void load_run(const uint16_t* src, int left, float (&v)[R]) {
    uint32_t w[R / 2];
#pragma unroll
    for (int e = 0; e < R / 2; ++e) w[e] = 0u;
    if (left >= R) {
        if constexpr (R == 4) {
            const u32x2 o = *reinterpret_cast<const u32x2_align2*>(src);
            w[0] = o[0]; w[1] = o[1];
        } else {
            const u32x4 o = *reinterpret_cast<const u32x4_align2*>(src);
            w[0] = o[0]; w[1] = o[1]; w[2] = o[2]; w[3] = o[3];
        }
    } else if (left > 0) {
        uint32_t x[R - 1];
#pragma unroll
        for (int e = 0; e < R - 1; ++e) x[e] = src[min(e, left - 1)];
#pragma unroll
        for (int e = 0; e < R - 1; ++e) w[e >> 1] |= e < left ? x[e] << (16 * (e & 1)) : 0u;
    }
#pragma unroll
    for (int e = 0; e < R / 2; ++e) {
        v[2 * e] = __builtin_bit_cast(float, w[e] << 16);
        v[2 * e + 1] = __builtin_bit_cast(float, w[e] & 0xFFFF0000u);
    }
}

// ---- activations (32 bits; hardware exp2 and reciprocal, 1 ulp each, for results that are rounded to bf16 or summed) ----
__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * z));
}
// The normal distribution's cdf, from formula 7.1.26 of Abramowitz and Stegun (erf to 1.5e-7, absolute), and exp(-z^2/2).
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.707106781f, fabsf(z), 1.f));
    e = __builtin_amdgcn_exp2f(-0.72134752f * z * z);
    float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
    p = __builtin_fmaf(p, t, 1.421413741f);
    p = __builtin_fmaf(p, t, -0.284496736f);
    p = __builtin_fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * e;
    return z < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float act_one(float z, int kind) {
    if (kind == QG_ACT_SILU) return z * sigmoid(z);
    if (kind == QG_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if (kind == QG_ACT_RELU) return z < 0.f ? 0.f : z;      // (NaN stays)
    return z;
}
// act(z) and its derivative
__device__ __forceinline__ float act_grad(float z, int kind, float& a) {
    if (kind == QG_ACT_SILU) {
        const float s = sigmoid(z);
        a = z * s;
        return __builtin_fmaf(a, 1.f - s, s);
    }
    if (kind == QG_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        a = z * c;
        return __builtin_fmaf(0.398942280f * z, e, c);
    }
    if (kind == QG_ACT_RELU) {
        a = z < 0.f ? 0.f : z;
        return z > 0.f ? 1.f : 0.f;
    }
    a = z;
    return 1.f;
}

// ---- epilogues that take runs of a row: a wave's blocks go through LDS one by one (as in store_block), a lane then has 8
// consecutive elements of a row, of both products for a pair, and memory is accessed in 16-byte runs.
template <typename E>
struct RunEpilogue : E {
    static constexpr int kStep = E::kPair ? 2 : 1;
    template <bool EXACT, int MB, int NB>
    __device__ __forceinline__ void tile(const f32x16 (&acc)[MB][NB], float* tp, int row0, int col0, bool inside, int M, int N,
                                         int lane) const {
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
            for (int b = 0; b < NB; b += kStep) {
#pragma unroll
                for (int p = 0; p < kStep; ++p)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        tp[p * kTransposeFloats + (8 * (v >> 2) + 4 * (lane >> 5) + (v & 3)) * kTransposePitch + (lane & 31)] =
                            acc[a][b + p][v];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = 16 * i + lane / 4, c = 8 * (lane % 4);
                    const int row = row0 + a * 32 + r, col = col0 + (b / kStep) * 32 + c;
                    const int left = EXACT || inside ? 8 : (row < M ? N - col : 0);
                    float v[kStep][8];
#pragma unroll
                    for (int p = 0; p < kStep; ++p) {
                        const float* src = tp + p * kTransposeFloats + r * kTransposePitch + c;
                        const f32x4 lo = *reinterpret_cast<const f32x4*>(src), hi = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[p][e] = lo[e];
                            v[p][4 + e] = hi[e];
                        }
                    }
                    if (left > 0) {
                        if constexpr (E::kPair) this->run(row, col, left, v[0], v[1]);
                        else this->run(row, col, left, v[0]);
                    }
                }
            }
    }
};

// z = sum + bias, y = act(z) + residual; z and residual may be missing.
struct ActRun {
    static constexpr bool kPair = false, kCounted = false;
    const uint16_t *bias, *residual;
    uint16_t *z, *y;
    int64_t ldc;
    int kind;
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&v)[R]) const {
        const int64_t at = (int64_t)row * ldc + col;
        float t[R];
        if (bias != nullptr) {
            load_run(bias + col, left, t);
#pragma unroll
            for (int e = 0; e < R; ++e) v[e] += t[e];
        }
        if (z != nullptr) store_run(z + at, left, v);
#pragma unroll
        for (int e = 0; e < R; ++e) v[e] = act_one(v[e], kind);
        if (residual != nullptr) {
            load_run(residual + at, left, t);
#pragma unroll
            for (int e = 0; e < R; ++e) v[e] += t[e];
        }
        store_run(y + at, left, v);
    }
};

// y = act(g) * u; g and u are stored where the backward pass will want them.
struct GatedRun {
    static constexpr bool kPair = true, kCounted = false;
    uint16_t *zg, *zu, *y;
    int64_t ldc;
    int kind;
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&g)[R], float (&u)[R]) const {
        const int64_t at = (int64_t)row * ldc + col;
        if (zg != nullptr) {
            store_run(zg + at, left, g);
            store_run(zu + at, left, u);
        }
#pragma unroll
        for (int e = 0; e < R; ++e) g[e] = act_one(g[e], kind) * u[e];
        store_run(y + at, left, g);
    }
};

// ---- kernels ----
enum : int { kDimM = 0, kDimN = 1 };
// Contraction of a part where the number of tiles is known to the device only: about two workgroups per CU for `live` tiles of a
// contraction of k, parts of `least` (a multiple of 64) and more.
__device__ __forceinline__ int live_chunk(int least, int k, int live) {
    const int splits = max(512 / live, 1);
    return max(least, ((k + splits - 1) / splits + 63) / 64 * 64);
}
template <typename OPB, typename EPI>
struct EpiProduct {
    LinOperand A, A2;
    OPB B, B2;
    EPI epi;
    int M, N, K, tiles_m, tiles_n;
    // An extent that only the device knows: *count rows or columns, at most M or N, and a multiple of `unit` (at
    // least 64: a whole number of steps; tiles are taken to be whole if unit is so many of them).  The grid is the largest one's;
    // the rest ends at once.
    const int32_t* count = nullptr;
    int dim = kDimM, unit = 0;
    // The contraction over `splits` workgroups per tile (blockIdx.y): `k_chunk` of it each (a multiple of 64), epi.split(s) for the
    // s-th one.
    int splits = 1, k_chunk = 0;
    int live_k = 0;      // > 0: the parts are live_chunk(k_chunk, live_k, tiles there are), the workgroups of further ones end at once
};

template <int AL, int BL, bool EXACT, int MB, int TN, int BK, int WM, bool DEEP, int KG, int TERMS, typename OPB, typename EPI>
__global__ __launch_bounds__(WM * 128 * KG, KG > 1 ? (MB == 1 ? 4 : 2) : WM == 2 ? 2 : 1) void k_gemm_epilogue(EpiProduct<OPB, EPI> p) {
    __shared__ __attribute__((aligned(16))) uint16_t smem[KG * TileGemm<AL, BL, MB, TN, BK, WM, KG>::SMEM];
    uint32_t grid = gridDim.x;
    if constexpr (EPI::kCounted) {
        if (p.count != nullptr) {
            const int n = *p.count;
            if (p.dim == kDimM) p.tiles_m = ((p.M = n) + 32 * MB * WM - 1) / (32 * MB * WM);
            else p.tiles_n = ((p.N = n) + TN - 1) / TN;
            grid = (uint32_t)(p.tiles_m * p.tiles_n + 7) / 8 * 8;      // the XCDs share what there is
            if (blockIdx.x >= grid) return;
        }
        if (p.splits > 1) {
            if (p.live_k > 0) p.k_chunk = live_chunk(p.k_chunk, p.live_k, p.tiles_m * p.tiles_n);
            const int k0 = (int)blockIdx.y * p.k_chunk;
            if (k0 >= p.K) return;
            auto at = [&](LinOperand& op, auto layout) {
                constexpr int L = decltype(layout)::value;
                static_assert(L == kBf16KFast || L == kBf16KSlow || L == kInt8KSlow, "others: not needed so far");
                const int64_t off = L == kBf16KFast ? k0 : k0 * op.ld;
                if constexpr (L == kInt8KSlow) {
                    op.base = static_cast<const int8_t*>(op.base) + off;
                    op.scales += (int64_t)k0 * op.sgroups;
                } else {
                    op.base = static_cast<const uint16_t*>(op.base) + off;
                }
            };
            at(p.A, std::integral_constant<int, AL>());
            at(p.B, std::integral_constant<int, BL>());
            if constexpr (TERMS == 2) {
                at(p.A2, std::integral_constant<int, AL>());
                at(p.B2, std::integral_constant<int, BL>());
            }
            p.K = min(p.k_chunk, p.K - k0);
            p.epi.split((int)blockIdx.y);
        }
    }
    const uint32_t tile = xcd_tile(blockIdx.x, grid);
    if (tile >= (uint32_t)(p.tiles_m * p.tiles_n)) return;
    tile_gemm_epi<AL, BL, EXACT, MB, TN, BK, WM, DEEP, KG, TERMS>(p.A, p.B, p.A2, p.B2, p.epi, p.M, p.N, p.K, p.tiles_m, p.tiles_n, tile,
                                                                  smem);
}

template <int AL, int BL, bool EXACT, int KW, typename OPB, typename EPI>
__global__ __launch_bounds__(64 * KW) void k_ksplit_epilogue(EpiProduct<OPB, EPI> p) {
    __shared__ __attribute__((aligned(16))) uint16_t smem[KSplit<AL, BL, KW, EPI::kPair ? 2 : 1>::SMEM];
    const uint32_t tile = xcd_tile(blockIdx.x, gridDim.x);
    if (tile >= (uint32_t)(p.tiles_m * p.tiles_n)) return;
    ksplit_epi<AL, BL, EXACT, KW>(p.A, p.B, p.epi, p.M, p.N, p.K, p.tiles_m, p.tiles_n, tile, smem);
}

// A part of a split contraction, in fp32: sum[split][row][col], rows `ld` (a multiple of 8) apart.
struct PartRun {
    static constexpr bool kPair = false, kCounted = true;
    float* sum;
    int64_t ld, stride;
    __device__ void split(int s) { sum += s * stride; }
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&v)[R]) const {
        float* p = sum + (int64_t)row * ld + col;
#pragma unroll
        for (int e = 0; e < R; e += 4)
            if (e < left) *reinterpret_cast<f32x4*>(p + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    }
};

// The parts added in order (times *scale), rounded once: out[row][col], or out[to[row]][col] where `to` is given and not negative.
// rows: *count of them where that is given.  live.k > 0: as many parts as live_chunk made of that many rows.
struct LiveParts {
    int k = 0, chunk = 0, side = 0, across = 0;      // side: of a tile; across: tiles per row of tiles
};
static __global__ __launch_bounds__(256) void k_join_parts(const float* __restrict__ sum, int64_t ld, int64_t stride, int splits,
                                                           LiveParts live, const int32_t* __restrict__ to, const int32_t* __restrict__ count,
                                                           const float* __restrict__ scale, int rows, int cols,
                                                           uint16_t* __restrict__ out, int64_t ld_out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, chunks = (cols + 7) / 8, row = i / chunks;
    const int there = count != nullptr ? *count : rows;
    if (row >= there) return;
    if (live.k > 0) {
        const int chunk = live_chunk(live.chunk, live.k, (there + live.side - 1) / live.side * live.across);
        splits = (live.k + chunk - 1) / chunk;
    }
    const int at = to != nullptr ? to[row] : (int)row, col = (int)(i - row * chunks) * 8;
    if (at < 0) return;
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    const float* p = sum + row * ld + col;
#pragma unroll 4
    for (int s = 0; s < splits; ++s, p += stride) {
        a += reinterpret_cast<const f32x4*>(p)[0];
        b += reinterpret_cast<const f32x4*>(p)[1];
    }
    const float f = scale != nullptr ? *scale : 1.f;
    const float v[8] = {f * a[0], f * a[1], f * a[2], f * a[3], f * b[0], f * b[1], f * b[2], f * b[3]};
    store_run(out + (int64_t)at * ld_out + col, cols - col, v);
}
static int launch_join_parts(const float* sum, int64_t ld, int64_t stride, int splits, LiveParts live, const int32_t* to, const int32_t* count,
                             const float* scale, int64_t rows, int64_t cols, uint16_t* out, int64_t ld_out, hipStream_t st) {
    hipLaunchKernelGGL(k_join_parts, dim3((unsigned)((rows * ((cols + 7) / 8) + 255) / 256)), dim3(256), 0, st, sum, ld, stride, splits, live, to,
                       count, scale, (int)rows, (int)cols, out, ld_out);
    return check_launch();
}

// One product (TERMS == 2: the sum of two of one shape) by tiles of TM = 32 MB WM rows and TN columns (a pair: TN / 2 of each).
template <int AL, int BL, int MB, int TN, int BK, int WM, bool DEEP_EXACT, bool DEEP_RAGGED, int KG, int TERMS, typename OPB, typename EPI>
static int launch_epilogue_shape(EpiProduct<OPB, EPI> p, hipStream_t st) {
    constexpr int TM = 32 * MB * WM, TC = EPI::kPair ? TN / 2 : TN;
    p.tiles_m = (p.M + TM - 1) / TM;
    p.tiles_n = (p.N + TC - 1) / TC;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    if (tiles * (WM * 128 * KG) >= (int64_t(1) << 32)) return QG_ERR_SHAPE;   // threads of one launch
    const unsigned grid = (unsigned)((tiles + 7) / 8 * 8);
    const int M = p.count != nullptr && p.dim == kDimM ? p.unit : p.M, N = p.count != nullptr && p.dim == kDimN ? p.unit : p.N;
    const bool exact = M % TM == 0 && N % TC == 0 && p.K % BK == 0 && p.A.ld % 8 == 0 && p.B.ld % 16 == 0;
    if (exact)
        hipLaunchKernelGGL((k_gemm_epilogue<AL, BL, true, MB, TN, BK, WM, DEEP_EXACT, KG, TERMS, OPB, EPI>), dim3(grid, p.splits),
                           dim3(128 * WM * KG), 0, st, p);
    else
        hipLaunchKernelGGL((k_gemm_epilogue<AL, BL, false, MB, TN, BK, WM, DEEP_RAGGED, KG, TERMS, OPB, EPI>), dim3(grid, p.splits),
                           dim3(128 * WM * KG), 0, st, p);
    return check_launch();
}

// 32 x 32 output elements per workgroup, the contraction over KW waves (see KSplit).
template <int AL, int BL, int KW, typename OPB, typename EPI>
static int launch_epilogue_ksplit(EpiProduct<OPB, EPI> p, hipStream_t st) {
    p.tiles_m = (p.M + 31) / 32;
    p.tiles_n = (p.N + 31) / 32;
    const unsigned grid = (unsigned)((p.tiles_m * p.tiles_n + 7) / 8 * 8);
    const bool exact = p.M % 32 == 0 && p.N % 32 == 0 && p.K % 64 == 0 && p.A.ld % 8 == 0 && p.B.ld % 16 == 0;
    if (exact) hipLaunchKernelGGL((k_ksplit_epilogue<AL, BL, true, KW, OPB, EPI>), dim3(grid), dim3(64 * KW), 0, st, p);
    else hipLaunchKernelGGL((k_ksplit_epilogue<AL, BL, false, KW, OPB, EPI>), dim3(grid), dim3(64 * KW), 0, st, p);
    return check_launch();
}

}  // namespace qg
