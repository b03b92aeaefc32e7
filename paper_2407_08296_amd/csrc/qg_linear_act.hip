// The INT8 linear layer with an epilogue (bias, activation, residual), and the gated pair of layers that opens a decoder's
// feed-forward block, with their backward passes.
//     act forward:     z = x W^T + bias,  y = act(z) + residual
//     act backward:    dz = dy act'(z),   dx = dz W,  G = dz^T x,  dbias = sum over tokens of dz
//     gated forward:   y = act(x Wg^T) * (x Wu^T)
//     gated backward:  dzg = dy zu act'(zg),  dzu = dy act(zg),  dx = dzg Wg + dzu Wu,  Gg = dzg^T x,  Gu = dzu^T x
// W is dequantized while it is staged, as in the plain layer.  The forward passes are one launch: the activation is applied to
// the fp32 sums, and z is rounded only where it is stored for the backward pass.  dz goes through the workspace, made by one pass over dy
// and z, in rows of whole cache lines whatever m is.  It is rounded to bf16 there, as an operand of two bf16 products: dx and G are then
// off by 0.0023 of their norm where their own rounding alone gives 0.0017.  dbias takes dz in fp32.
#include "qg_epilogue.h"

namespace qg {

static bool all_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (!aligned16(p)) return false;
    return true;
}

// ---- dz: 8 columns of a row per thread, LANES threads per row.  Bound by HBM (6 bytes per element, a pair 10).  dbias: the columns'
// sums over a slab from registers, a wave's rows by lane swaps, the four waves added in order, slabs added by k_column_sums.
// LANES = 64: 512 columns and every 4th row of a slab per wave.  LANES = 2: 16 columns and all rows, so that dbias takes no
// second kernel and short batches reach all CUs (256 x 2048, gelu and dbias, us: 7.1, 8.9 with two kernels, 8.5 with 64 columns
// per workgroup).  A pair of 4096 x 11008: 83 us (5.4 TB/s), of 1000 x 5461 (unaligned rows) 15 (3.6 TB/s).
template <bool PAIR, int LANES>
__global__ __launch_bounds__(LANES == 2 ? 512 : 256) void k_act_backward(const uint16_t* __restrict__ dy, const uint16_t* __restrict__ zg,
                                                      const uint16_t* __restrict__ zu, uint16_t* __restrict__ dzg,
                                                      uint16_t* __restrict__ dzu, float* __restrict__ part, int tokens, int m, int64_t ld,
                                                      int64_t ld_out, int rows, int kind) {
    constexpr int NT = LANES == 2 ? 512 : 256, WAVES = NT / 64, STEP = NT / LANES;          // rows at a time
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * (8 * LANES) + lane * 8, left = m - col;
    const int first = blockIdx.y * rows, last = min(first + rows, tokens);
    float sum[8] = {};
    auto fetch = [&](int t, float (&d)[8], float (&z)[8], float (&u)[8]) {
        const int64_t at = (int64_t)t * ld + col;
        load_run(dy + at, left, d);
        if (PAIR || kind != QG_ACT_NONE) load_run(zg + at, left, z);
        if constexpr (PAIR) load_run(zu + at, left, u);
    };
    auto use = [&](int t, const float (&d)[8], const float (&z)[8], const float (&u)[8]) {
        const int64_t to = (int64_t)t * ld_out + col;
        float o[8], p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a;
            const float g = kind == QG_ACT_NONE && !PAIR ? 1.f : act_grad(z[e], kind, a);
            if constexpr (PAIR) {
                o[e] = d[e] * u[e] * g;
                p[e] = d[e] * a;
            } else {
                o[e] = d[e] * g;
                sum[e] += o[e];
            }
        }
        if (PAIR || dzg != nullptr) store_run(dzg + to, 8, o);        // (a row's last chunk is whole: zeros past its end)
        if constexpr (PAIR) store_run(dzu + to, 8, p);
    };
    if (left > 0) {
        int t = first + sub;
        float d[2][8], z[2][8], u[2][8];
        for (; t + STEP < last; t += 2 * STEP) {      // two rows on their way at once
            fetch(t, d[0], z[0], u[0]);
            fetch(t + STEP, d[1], z[1], u[1]);
            use(t, d[0], z[0], u[0]);
            use(t + STEP, d[1], z[1], u[1]);
        }
        if (t < last) {
            fetch(t, d[0], z[0], u[0]);
            use(t, d[0], z[0], u[0]);
        }
    }
    if (PAIR || part == nullptr) return;
    __shared__ float sums[WAVES][8 * LANES];
    if constexpr (LANES == 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int off = 2; off < 64; off <<= 1) sum[e] += __shfl_xor(sum[e], off, 64);
    }
    if ((threadIdx.x & 63) < LANES)
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[wave][e * LANES + lane] = sum[e];
    __syncthreads();
    if (threadIdx.x >= LANES || left <= 0) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum[e] += sums[w][e * LANES + lane];
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

// Rows of a slab, and slabs: about a thousand workgroups of 64 lanes per row where there are rows for them.
struct Slabs {
    int rows, count;
};
static Slabs act_slabs(int64_t tokens, int64_t m) {
    const int64_t across = (m + 511) / 512, want = (1024 + across - 1) / across;
    int64_t rows = (tokens + want - 1) / want;
    rows = (rows + 3) / 4 * 4;
    return {(int)rows, (int)((tokens + rows - 1) / rows)};
}
// dbias in one kernel: up to 2048 tokens (a workgroup takes all of them) and 2^21 elements (beyond, 16 columns of a row per workgroup
// read worse than the second kernel costs).  The whole backward pass, us, one / two kernels: 32 x 768 columns 17.0 / 19.3, 1024 x 256
// 16.7 / 19.4, 768 x 2048 30.1 / 32.2, 1024 x 2048 32.7 / 34.2, 2048 x 1024 39.6 / 40.2; but 4096 x 64 35.3 / 34.2, 512 x 8192
// 84 / 81, 1024 x 4096 51.9 / 48.8, 1024 x 8192 147 / 133.
static bool act_one_slab(int64_t tokens, int64_t m) { return tokens <= 2048 && tokens * m <= (int64_t(1) << 21); }

// part: one row of sums per slab, or dbias itself where there is one slab (a pair has no dbias)
template <bool PAIR>
static int launch_act_backward(const uint16_t* dy, const uint16_t* zg, const uint16_t* zu, uint16_t* dzg, uint16_t* dzu, float* part,
                               float* dbias, int64_t tokens, int64_t m, int64_t ld, int64_t ld_out, int kind, hipStream_t st) {
    if constexpr (!PAIR) {
        if (dbias != nullptr && act_one_slab(tokens, m)) {
            hipLaunchKernelGGL((k_act_backward<false, 2>), dim3((unsigned)((m + 15) / 16)), dim3(512), 0, st, dy, zg, zu, dzg, dzu, dbias,
                               (int)tokens, (int)m, ld, ld_out, (int)tokens, kind);
            return check_launch();
        }
    }
    const Slabs s = act_slabs(tokens, m);
    hipLaunchKernelGGL((k_act_backward<PAIR, 64>), dim3((unsigned)((m + 511) / 512), (unsigned)s.count), dim3(256), 0, st, dy, zg, zu, dzg,
                       dzu, dbias != nullptr ? part : nullptr, (int)tokens, (int)m, ld, ld_out, s.rows, kind);
    if constexpr (!PAIR) {
        if (dbias != nullptr)
            hipLaunchKernelGGL(k_column_sums, dim3((unsigned)((m + 63) / 64)), dim3(1024), 0, st, part, s.count, (int)m, dbias);
    }
    return check_launch();
}

// Tiles of the products with an epilogue, x W^T of one weight: those of the plain layer's forward pass (see launch_tile_gemm, which
// has the measurements on both sides of each rule), but for its direct loads of whole 256 x 256 tiles: two register sets are ahead of
// them here (4096 tokens, 4096 -> 11008, us: 417 / 456, the gated pair 778 / 885).
template <typename EPI>
static int launch_act_forward(EpiProduct<LinOperand, EPI> p, hipStream_t st) {
    constexpr int AL = kBf16KFast, BL = kInt8KFast;
    if (lin_ksplit<AL, BL>(p.M, p.N, p.K, 0)) {
        const int64_t t32 = (int64_t)((p.M + 31) / 32) * ((p.N + 31) / 32);
        return t32 <= 256 ? launch_epilogue_ksplit<AL, BL, 8>(p, st) : launch_epilogue_ksplit<AL, BL, 4>(p, st);
    }
    auto tiles = [&](int tm, int tn) { return (int64_t)((p.M + tm - 1) / tm) * ((p.N + tn - 1) / tn); };
    const bool small = lin_small<AL, BL>(p.M, p.N, 1);
    if (p.K >= 512) {      // two groups of waves per tile while tiles are about a workgroup per CU or fewer
        if (!small) {
            if (p.K >= 768 && tiles(128, 128) <= 256) return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, true, true, 2, 1>(p, st);
        } else if (tiles(64, 64) <= 256) {
            return launch_epilogue_shape<AL, BL, 1, 64, 64, 2, true, true, 2, 1>(p, st);
        } else if (tiles(128, 64) <= 256 && p.K >= (p.K % 16 != 0 ? 4096 : p.K % 64 == 0 ? 640 : 960)) {
            return launch_epilogue_shape<AL, BL, 2, 64, 64, 2, true, true, 2, 1>(p, st);
        }
    }
    if (p.M >= 1024 && tiles(256, 256) >= 256) return launch_epilogue_shape<kBf16KFast, kInt8KFast, 2, 256, 64, 4, true, true, 1, 1>(p, st);
    if (small) return launch_epilogue_shape<AL, BL, 1, 64, 64, 2, true, true, 1, 1>(p, st);
    if (tiles(128, 128) > 256 && tiles(128, 128) <= 512) return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, false, false, 1, 1>(p, st);
    return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, true, true, 1, 1>(p, st);
}

// ... of a pair: N columns of each, the tile's columns shared between the two so that x is staged once for both.  4096 tokens, 4096 -> 2 x
// 11008: 727 to 755 us from card to card (1016 to 978 TFLOP/s; without zg and zu 9 % less: their stores come at the end of a tile, when the
// CU's matrix pipe is idle); 256 tokens 80 us; one token 26.6 us (3.4 TB/s of codes; a kernel that loads them straight into matrix operands,
// without LDS, took 25.9 to 30).
// Tiles, us, by what the rule takes / the next one (T32: blocks of 32 x 32 columns of each; T64, T128: tiles of 64 or 128 tokens by 64):
//  * the contraction over waves up to T32 = 512: 64 tokens, 4096 -> 8192 (512) 26.8 / 28.5, 64 tokens, 1024 -> 5461 (342) 8.7 / 10.3, but
//    150 tokens, 2047 -> 4095 (640) 38.5 / 24.0, 64 tokens, 4096 -> 11008 (688) 40 / 30.
//  * 64 tokens in two groups of waves up to T64 = 256: 128 tokens, 4096 -> 8192 (256) 30.7, 128 tokens a tile 42.7 to 47; one
//    group below K = 1024: 500 tokens, 768 -> 2048 11.5 / 12.2, at 1024 (300 tokens, 2736 columns) 12.3 / 12.2, at 1536 16.4 / 14.2.
//  * 128 tokens in two groups up to T128 = 256: 500 tokens, 2048 -> 4096 (256) 28.0, one group 29.6, 150 tokens, 4096 -> 8192 49.4 / 52.5;
//    one group below K = 768: 500 tokens, 512 -> 4096 12.8 / 12.5.
//  * 64 tokens, one group, up to T64 = 512: 700 tokens, 2048 -> 2736 (473) 31.1, 128 tokens a tile 40.0; 700 tokens, 1024 -> 2736
//    18.4 / 24.2; not beyond: 256 tokens, 4096 -> 11008 (688) 91 / 75, 1000 tokens, 2048 -> 5461 (1376) 87 / 68.
//  * 256 tokens from a workgroup per CU on, as for one weight.
template <typename EPI>
static int launch_gated_forward(EpiProduct<LinPairOperand, EPI> p, hipStream_t st) {
    constexpr int AL = kBf16KFast, BL = kInt8KFast;
    auto tiles = [&](int tm, int tn) { return (int64_t)((p.M + tm - 1) / tm) * ((p.N + tn - 1) / tn); };
    const int64_t t32 = tiles(32, 32), t64 = tiles(64, 64), t128 = tiles(128, 64);
    if (t32 <= 256) return launch_epilogue_ksplit<AL, BL, 8>(p, st);
    if (t32 <= 512) return launch_epilogue_ksplit<AL, BL, 4>(p, st);
    if (t64 <= 256 && p.K >= 1024) return launch_epilogue_shape<AL, BL, 1, 128, 64, 2, true, true, 2, 1>(p, st);
    if (t64 > 256 && t128 <= 256 && p.K >= 768) return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, true, true, 2, 1>(p, st);
    if (t64 <= 256 || (t128 > 256 && t64 <= 512)) return launch_epilogue_shape<AL, BL, 1, 128, 64, 2, true, true, 1, 1>(p, st);
    if (p.M >= 1024 && tiles(256, 128) >= 256) return launch_epilogue_shape<AL, BL, 2, 256, 64, 4, true, true, 1, 1>(p, st);
    return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, true, true, 1, 1>(p, st);
}

// dx = dzg Wg + dzu Wu, tokens x n, one accumulator for both.  Fewer than 512 tiles of 128 x 128 (two per CU): both contractions split
// over workgroups, parts of 512 at least, in fp32 through the workspace.  1000 tokens, 2 x 5461 -> 2048, us: 68 and 7 for the sum of
// four parts, 110 in 64 x 64 tiles that take the whole contraction (the pass: 149, 155 and 161 with parts for one and for four
// workgroups per CU; 256 tokens, 2 x 11008 -> 4096 170, 172, 180; 1400 tokens, 2 x 5461 -> 2048 200, 210, 197); 4096 tokens, 2 x 11008
// -> 4096 700 (1055 TFLOP/s).  Ragged 256 x 256 tiles hold 233 registers of a lane in scratch for the checks of two products beside two
// register sets; with dz, 4000 tokens take 763 us like 4096 with 781 (3840, which are 240 of these tiles and go by 128 x 128, 898).
static int64_t gated_dx_chunk(int64_t tokens, int64_t m, int64_t n) {
    const int64_t t128 = ((tokens + 127) / 128) * ((n + 127) / 128), room = 512 / t128, most = m / 512, splits = room < most ? room : most;
    return splits <= 1 ? m : ((m + splits - 1) / splits + 63) / 64 * 64;
}
static int launch_gated_dx(const LinOperand& dzg, const LinOperand& dzu, const LinOperand& Wg, const LinOperand& Wu, uint16_t* dx, int64_t ld,
                           int64_t tokens, int64_t m, int64_t n, float* parts, hipStream_t st) {
    const int64_t chunk = gated_dx_chunk(tokens, m, n);
    if (chunk < m) {
        const int64_t ldp = (n + 7) / 8 * 8;
        EpiProduct<LinOperand, RunEpilogue<PartRun>> p;
        p.A = dzg, p.A2 = dzu, p.B = Wg, p.B2 = Wu;
        static_cast<PartRun&>(p.epi) = PartRun{parts, ldp, tokens * ldp};
        p.M = (int)tokens, p.N = (int)n, p.K = (int)m;
        p.k_chunk = (int)chunk;
        p.splits = (int)((m + chunk - 1) / chunk);
        if (int e = launch_epilogue_shape<kBf16KFast, kInt8KSlow, 2, 128, 64, 2, true, true, 1, 2>(p, st)) return e;
        return launch_join_parts(parts, ldp, tokens * ldp, p.splits, {}, nullptr, nullptr, nullptr, tokens, n, dx, ld, st);
    }
    EpiProduct<LinOperand, PlainEpilogue<uint16_t>> p;
    p.A = dzg, p.A2 = dzu, p.B = Wg, p.B2 = Wu;
    p.epi = PlainEpilogue<uint16_t>{nullptr, dx, ld};
    p.M = (int)tokens, p.N = (int)n, p.K = (int)m;
    if (p.M >= 1024 && (int64_t)((p.M + 255) / 256) * ((p.N + 255) / 256) >= 256)
        return launch_epilogue_shape<kBf16KFast, kInt8KSlow, 2, 256, 64, 4, true, true, 1, 2>(p, st);
    return launch_epilogue_shape<kBf16KFast, kInt8KSlow, 2, 128, 64, 2, true, true, 1, 2>(p, st);
}

// Rows of x at a pitch of whole 16-byte chunks, zeros past their ends.
__global__ __launch_bounds__(256) void k_align_rows(const uint16_t* __restrict__ x, int64_t ld, int rows, int cols, uint16_t* __restrict__ out,
                                                    int64_t pitch) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, chunks = pitch / 8, row = i / chunks;
    if (row >= rows) return;
    const int col = (int)(i - row * chunks) * 8;
    float v[8];
    load_run(x + row * ld + col, cols - col, v);
    store_run(out + row * pitch + col, 8, v);
}

// G = dz^T x for one or two dz of rows `ldz` apart (a multiple of 8).  Direct loads where there are tiles of 128 x 256 for every CU; they
// want rows that start on 16 bytes, and x is copied to such where it has others (600 tokens, 2997 and 2 x 6869, us: 97 and 5 for the
// copy; without direct loads 130).  1000 tokens, 2 x 5461 x 2048: both in one launch 54 us, in two of other tiles 91; 4096 tokens, 2 x 11008
// x 4096 683 (1080 TFLOP/s).
// (Rows longer than that kernel addresses: the other tiles.)
static int64_t dz_pitch(int64_t m) { return (m + 63) / 64 * 64; }
static bool grad_w_direct(int64_t m, int64_t n, int64_t ld_n, int count) {
    return ((m + kLinTM - 1) / kLinTM) * ((n + 255) / 256) * count >= 256 && dz_pitch(m) <= kKSlowPitch && (ld_n + 7) / 8 * 8 <= kKSlowPitch;
}
static size_t grad_w_copy_bytes(int64_t tokens, int64_t m, int64_t n, int count) {   // of x, whatever its pitch turns out to be
    return grad_w_direct(m, n, n, count) && n % 8 != 0 ? (size_t)tokens * ((n + 7) / 8 * 8) * 2 : 0;
}
static int launch_act_grad_w(const uint16_t* dz, const uint16_t* dz2, int64_t ldz, const uint16_t* x, int64_t ld_n, uint16_t* G, uint16_t* G2,
                             int64_t tokens, int64_t m, int64_t n, uint16_t* copy, hipStream_t st) {
    const int count = dz2 != nullptr ? 2 : 1;
    if (grad_w_direct(m, n, ld_n, count)) {
        int64_t ldx = ld_n;
        if (ld_n % 8 != 0) {
            ldx = (n + 7) / 8 * 8;
            hipLaunchKernelGGL(k_align_rows, dim3((unsigned)((tokens * (ldx / 8) + 255) / 256)), dim3(256), 0, st, x, ld_n, (int)tokens, (int)n,
                               copy, ldx);
            x = copy;
        }
        const int64_t tiles_m = (m + kLinTM - 1) / kLinTM, tiles_n = (n + 255) / 256;
        const dim3 grid((unsigned)((tiles_m * tiles_n + 7) / 8 * 8), (unsigned)count);
        const KSlowOut out = {(int)m, (int)n, ld_n, nullptr, dz2, G2, nullptr};
        hipLaunchKernelGGL((k_gemm_kslow_direct<uint16_t, true>), grid, dim3(256), 0, st, dz, x, G, (int)ldz, (int)ldx, (int)tokens, (int)tiles_m,
                           (int)tiles_n, out);
        return check_launch();
    }
    const LinOperand xo = {x, nullptr, ld_n, 0};
    for (int i = 0; i < count; ++i) {
        const LinOperand d = {i == 0 ? dz : dz2, nullptr, ldz, 0};
        if (int e = launch_linear_backward<kInt8KSlow>(d, xo, nullptr, tokens, n, m, ld_n, d, xo, i == 0 ? G : G2, m, n, tokens, ld_n, st)) return e;
    }
    return QG_OK;
}

static size_t whole_lines_of(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace qg

using namespace qg;

extern "C" int qg_int8_linear_act_forward(const uint16_t* x_bf16, const int8_t* Wq, const float* Ws, const uint16_t* bias_bf16,
                                          const uint16_t* residual_bf16, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n,
                                          int64_t ld_m, int group, uint16_t* z_bf16, uint16_t* y_bf16, void* stream) {
    if (!x_bf16 || !Wq || !Ws || !y_bf16) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_linear(tokens, m, n, group)) return e;
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

extern "C" size_t qg_int8_linear_act_workspace_bytes(int64_t tokens, int64_t m, int64_t n) {
    if (check_linear(tokens, m, n, kGroup)) return 0;
    return whole_lines_of((size_t)tokens * dz_pitch(m) * 2) + whole_lines_of((size_t)act_slabs(tokens, m).count * (size_t)m * 4) +
           grad_w_copy_bytes(tokens, m, n, 1);
}

extern "C" int qg_int8_linear_act_backward(const uint16_t* dy_bf16, const uint16_t* z_bf16, const uint16_t* x_bf16, const int8_t* Wq,
                                           const float* Ws, int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m,
                                           int group, uint16_t* dx_bf16, uint16_t* G_bf16, float* dbias, void* workspace,
                                           size_t workspace_bytes, void* stream) {
    if (!dy_bf16 || (!dx_bf16 && !G_bf16 && !dbias)) return QG_ERR_NULL;
    if ((dx_bf16 && (!Wq || !Ws)) || (G_bf16 && !x_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (act != QG_ACT_NONE && !z_bf16) return QG_ERR_NULL;
    if (int e = check_linear(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({dy_bf16, z_bf16, x_bf16, Wq, Ws, dx_bf16, G_bf16, dbias, workspace})) return QG_ERR_ALIGN;
    if ((dbias || act != QG_ACT_NONE) && (!workspace || workspace_bytes < qg_int8_linear_act_workspace_bytes(tokens, m, n)))
        return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    const bool products = dx_bf16 || G_bf16;
    const int64_t ldz = dz_pitch(m);
    uint16_t* dz = act != QG_ACT_NONE && products ? static_cast<uint16_t*>(workspace) : nullptr;
    float* part_at = dz || dbias ? reinterpret_cast<float*>(static_cast<char*>(workspace) + whole_lines_of((size_t)tokens * ldz * 2)) : nullptr;
    if (dz || dbias)
        if (int e = launch_act_backward<false>(dy_bf16, z_bf16, nullptr, dz, nullptr, part_at, dbias, tokens, m, ld_m, ldz, act, st)) return e;
    if (!products) return QG_OK;
    const LinOperand d = {dz ? dz : dy_bf16, nullptr, dz ? ldz : ld_m, 0}, x = {x_bf16, nullptr, ld_n, 0};
    const LinOperand W = {Wq, Ws, ld_n, (int)((n + kGroup - 1) / kGroup)};
    if (G_bf16 && dz && grad_w_direct(m, n, ld_n, 1)) {
        if (dx_bf16)
            if (int e = launch_linear_backward<kInt8KSlow>(d, W, dx_bf16, tokens, n, m, ld_n, d, x, nullptr, m, n, tokens, ld_n, st)) return e;
        char* copy = reinterpret_cast<char*>(part_at) + whole_lines_of((size_t)act_slabs(tokens, m).count * (size_t)m * 4);
        return launch_act_grad_w(dz, nullptr, ldz, x_bf16, ld_n, G_bf16, nullptr, tokens, m, n, reinterpret_cast<uint16_t*>(copy), st);
    }
    return launch_linear_backward<kInt8KSlow>(d, W, dx_bf16, tokens, n, m, ld_n, d, x, G_bf16, m, n, tokens, ld_n, st);
}

extern "C" int qg_int8_gated_forward(const uint16_t* x_bf16, const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus,
                                     int act, int64_t tokens, int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group,
                                     uint16_t* zg_bf16, uint16_t* zu_bf16, uint16_t* y_bf16, void* stream) {
    if (!x_bf16 || !Wgq || !Wgs || !Wuq || !Wus || !y_bf16 || (!zg_bf16 != !zu_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_linear(tokens, m, n, group)) return e;
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

extern "C" size_t qg_int8_gated_workspace_bytes(int64_t tokens, int64_t m, int64_t n) {
    if (check_linear(tokens, m, n, kGroup)) return 0;
    const int64_t chunk = gated_dx_chunk(tokens, m, n), splits = chunk < m ? (m + chunk - 1) / chunk : 0;
    return 2 * whole_lines_of((size_t)tokens * dz_pitch(m) * 2) + whole_lines_of((size_t)splits * tokens * ((n + 7) / 8 * 8) * 4) +
           grad_w_copy_bytes(tokens, m, n, 2);
}

extern "C" int qg_int8_gated_backward(const uint16_t* dy_bf16, const uint16_t* zg_bf16, const uint16_t* zu_bf16, const uint16_t* x_bf16,
                                      const int8_t* Wgq, const float* Wgs, const int8_t* Wuq, const float* Wus, int act, int64_t tokens,
                                      int64_t m, int64_t n, int64_t ld_n, int64_t ld_m, int group, uint16_t* dx_bf16, uint16_t* Gg_bf16,
                                      uint16_t* Gu_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    if (!dy_bf16 || !zg_bf16 || !zu_bf16 || (!Gg_bf16 != !Gu_bf16) || (!dx_bf16 && !Gg_bf16)) return QG_ERR_NULL;
    if ((dx_bf16 && (!Wgq || !Wgs || !Wuq || !Wus)) || (Gg_bf16 && !x_bf16)) return QG_ERR_NULL;
    if (act < QG_ACT_NONE || act > QG_ACT_GELU) return QG_ERR_SHAPE;
    if (int e = check_linear(tokens, m, n, group)) return e;
    if (int e = check_pitch(tokens > m ? tokens : m, n, ld_n)) return e;
    if (int e = check_pitch(tokens, m, ld_m)) return e;
    if (!all_aligned({dy_bf16, zg_bf16, zu_bf16, x_bf16, Wgq, Wgs, Wuq, Wus, dx_bf16, Gg_bf16, Gu_bf16, workspace})) return QG_ERR_ALIGN;
    if (!workspace || workspace_bytes < qg_int8_gated_workspace_bytes(tokens, m, n)) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t ldz = dz_pitch(m);
    const size_t dz_bytes = whole_lines_of((size_t)tokens * ldz * 2);
    uint16_t *dzg = static_cast<uint16_t*>(workspace), *dzu = dzg + dz_bytes / 2;
    float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * dz_bytes);
    if (int e = launch_act_backward<true>(dy_bf16, zg_bf16, zu_bf16, dzg, dzu, nullptr, nullptr, tokens, m, ld_m, ldz, act, st)) return e;
    const int sg = (int)((n + kGroup - 1) / kGroup);
    if (dx_bf16)
        if (int e = launch_gated_dx({dzg, nullptr, ldz, 0}, {dzu, nullptr, ldz, 0}, {Wgq, Wgs, ld_n, sg}, {Wuq, Wus, ld_n, sg}, dx_bf16, ld_n,
                                    tokens, m, n, parts, st))
            return e;
    if (!Gg_bf16) return QG_OK;
    const int64_t chunk = gated_dx_chunk(tokens, m, n), splits = chunk < m ? (m + chunk - 1) / chunk : 0;
    char* copy = reinterpret_cast<char*>(parts) + whole_lines_of((size_t)splits * tokens * ((n + 7) / 8 * 8) * 4);
    return launch_act_grad_w(dzg, dzu, ldz, x_bf16, ld_n, Gg_bf16, Gu_bf16, tokens, m, n, reinterpret_cast<uint16_t*>(copy), st);
}
