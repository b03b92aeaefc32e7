// Cross entropy of a language model's head over its vocabulary, without the logits in memory.  With x [T][h], W [V][h],
// z = x W^T:
//     lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,label
//     dl_tv = dloss_t (exp(z_tv - lse_t) - [v = label]),   dx = dl W,   dW = dl^T x
// rows:     the tokens that have a loss, put together: their rows of x, zeros up to a multiple of 256 of them, and how many there
//           are, which only the device knows.  Prompts and padding take no part from there on, and what they hold never meets a
//           product (0 times it would be NaN in dW if it is not finite).  What that saves comes in steps of the rows that are filled
//           up (1000 tokens, 2048 x 32003, both passes: 340 us with 497 of them learned, 464 with 523), and little of it in dx of a
//           large batch, whose tiles are chosen for all tokens.  4096 tokens, 4096 x 32000, us with 100 / 50 / 20 / 5 % of them
//           learned: forward 998 / 572 / 252 / 116, backward 2916 / 1965 / 1237 / 1060, of which dx 950 at 5 %.
// forward:  one product whose epilogue leaves, of every tile, each token's maximum and sum of exponentials over the tile's
//           entries, and the label's logit; a second kernel joins them.  The product is computed as W x^T, so that a lane's sums
//           belong to one token and most of the reduction stays in its registers.
// backward: the vocabulary in pieces.  For each, the logits are computed again with dl in the epilogue (bf16, the operand of the
//           two products), then dW's rows of the piece, and dx, which is added up over the pieces in fp32.
// dl is held relative to the largest |dloss|, which dx and dW are multiplied by in fp32: a mean's gradient at a label is then close to -1,
// which bf16 holds exactly, and not that fraction of 1/T, whose rounding every element of a row would share.
// Eight T V h flop against six with the logits kept; T x V numbers are never stored, only T x piece.
#include "qg_epilogue.h"

namespace qg {

constexpr float kLog2e = 1.44269504f;

// ---- forward ----
// 4096 tokens, 4096 x 32000: 930 us (up to 1000 from card to card; 1155 TFLOP/s, the matrix pipe busy 54 % of the time at 2.0 GHz); 256
// tokens, 768 x 32000: 20.5 us, of which W's bytes take 10; one token, 4096 x 32000: 51 us (5.1 TB/s).
// Rows of the product are vocabulary entries, columns tokens.  A lane has 16 entries of each block of its column's token, the lane 32
// further the other 16.
struct StatsEpilogue {
    static constexpr bool kPair = false, kCounted = true;
    const int32_t* label32;       // of the tokens put together, or
    const int64_t* labels;        // as the caller has them
    float* label_logit;
    f32x2* part;        // [slots][stride]: maximum and sum of exp(z - maximum) over a wave's 32 MB rows
    int64_t stride;
    __device__ void split(int) {}
    template <bool EXACT, int MB, int NB>
    __device__ __forceinline__ void tile(const f32x16 (&acc)[MB][NB], float*, int row0, int col0, bool inside, int M, int N,
                                         int lane) const {
        const int slot = row0 / (32 * MB), sub = 4 * (lane >> 5);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int col = col0 + b * 32 + (lane & 31);
            const bool token = EXACT || inside || col < N;
            int label = -1;
            if (token) {
                if (label32 != nullptr) label = label32[col];
                else if (const int64_t l = labels[col]; l >= 0 && l < M) label = (int)l;
            }
            const int at = label - row0 - sub;      // row of the label among the lane's
            float top = -INFINITY, z = 0.f;
            bool mine = false;
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = a * 32 + 8 * (v >> 2) + (v & 3);
                    if (EXACT || inside || row0 + sub + r < M) top = fmaxf(top, acc[a][b][v]);
                    if (at == r) {
                        z = acc[a][b][v];
                        mine = true;
                    }
                }
            if (mine) label_logit[col] = z;
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float ref = top == -INFINITY ? 0.f : top * kLog2e;
            float sum = 0.f;
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = a * 32 + 8 * (v >> 2) + (v & 3);
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[a][b][v], kLog2e, -ref));
                    sum += EXACT || inside || row0 + sub + r < M ? e : 0.f;
                }
            sum += __shfl_xor(sum, 32, 64);
            if (lane < 32 && token) part[(int64_t)slot * stride + col] = f32x2{top, sum};
        }
    }
};

// 16 tokens per workgroup, 64 slices of the slots: maxima first, then the sums below the token's maximum, in a fixed order.  4 to 6.5 us.
__global__ __launch_bounds__(1024) void k_head_join(const f32x2* __restrict__ part, int slots, int64_t stride,
                                                    const int64_t* __restrict__ labels, int64_t vocab,
                                                    const int32_t* __restrict__ rows, const float* __restrict__ label_logit,
                                                    const int32_t* __restrict__ count, int tokens, float* __restrict__ loss,
                                                    float* __restrict__ lse) {
    __shared__ float most[16][17], sums[16][17];
    if (count != nullptr) tokens = *count;
    if ((int)blockIdx.x * 16 >= tokens) return;
    const int lane = threadIdx.x & 15, slice = threadIdx.x >> 4, wave = threadIdx.x >> 6, t = blockIdx.x * 16 + lane;
    float top = -INFINITY, sum = 0.f;
    const bool mine = t < tokens;
    // slots of this slice, eight at a time: loads ahead of the exponentials
    for (int s0 = slice; s0 < slots; s0 += 512) {
        f32x2 p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = s0 + 64 * i;
            p[i] = mine && s < slots ? part[(int64_t)s * stride + t] : f32x2{-INFINITY, 0.f};
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) now = fmaxf(now, p[i][0]);
        const float ref = now == -INFINITY ? 0.f : now;
        sum *= __builtin_amdgcn_exp2f((top - ref) * kLog2e);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(p[i][1], __builtin_amdgcn_exp2f((p[i][0] - ref) * kLog2e), sum);
        top = now;
    }
    float all = fmaxf(top, __shfl_xor(top, 16, 64));      // the wave's four slices
    all = fmaxf(all, __shfl_xor(all, 32, 64));
    if ((threadIdx.x & 63) < 16) most[wave][lane] = all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) all = fmaxf(all, most[i][lane]);
    const float ref = all == -INFINITY ? 0.f : all;
    sum *= __builtin_amdgcn_exp2f((top - ref) * kLog2e);
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if ((threadIdx.x & 63) < 16) sums[wave][lane] = sum;
    __syncthreads();
    if (slice != 0 || !mine) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += sums[i][lane];
    const int row = rows != nullptr ? rows[t] : t;
    if (row < 0) return;
    const float l = all + logf(sum);
    const bool learned = rows != nullptr || (labels[t] >= 0 && labels[t] < vocab);
    lse[row] = learned ? l : 0.f;
    loss[row] = learned ? l - label_logit[t] : 0.f;
}

// ---- the tokens that have a loss ----
// Of each such token: its row of x, its number, its label in 32 bits and (backward) its lse and dloss; then rows of zeros up to a
// multiple of `unit`.  The others' loss and lse, or row of dx, become zero here.  A workgroup counts the labels for itself
// (they are few bytes and stay in the cache): one launch, and an order that does not depend on timing.  5 us and up: 1000 tokens of 2048
// 8 to 10, 4096 of 4096 27 (a copy of that size 14).
struct HeadRows {
    const uint16_t* x;
    const int64_t* labels;
    const float *lse_in, *dloss_in;      // backward only
    int64_t ld, vocab;
    int tokens, padded, unit, h, hp, per;   // padded: tokens up to a multiple of unit; per: tokens of a workgroup
    uint16_t* xc;
    int32_t *rows, *label32, *count;
    float *lse, *dloss, *scale;          // backward only; dloss: relative to *scale, the largest |dloss|
    float *loss_out, *lse_out;           // forward only
    uint16_t* dx;                        // backward only, may be NULL
};
__global__ __launch_bounds__(256) void k_head_rows(HeadRows a) {
    __shared__ int before_s[4], all_s[4];
    __shared__ float most_s[4];
    const int first = (int)blockIdx.x * a.per, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto learned = [&](int t) {
        const int64_t l = a.labels[t];
        return l >= 0 && l < a.vocab;
    };
    int before = 0, all = 0;
    float most = 0.f;
#pragma unroll 4
    for (int t = threadIdx.x; t < a.tokens; t += 256) {
        const int one = learned(t);
        all += one;
        before += t < first ? one : 0;
        if (a.scale != nullptr) most = fmaxf(most, one ? fabsf(a.dloss_in[t]) : 0.f);
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        all += __shfl_xor(all, off, 64);
        before += __shfl_xor(before, off, 64);
        most = fmaxf(most, __shfl_xor(most, off, 64));
    }
    if (lane == 0) {
        before_s[wave] = before;
        all_s[wave] = all;
        most_s[wave] = most;
    }
    __syncthreads();
    all = all_s[0] + all_s[1] + all_s[2] + all_s[3];
    before = before_s[0] + before_s[1] + before_s[2] + before_s[3];
    most = fmaxf(fmaxf(most_s[0], most_s[1]), fmaxf(most_s[2], most_s[3]));
    if (!(most > 0.f && most < INFINITY)) most = 1.f;
    // (rows of zeros where no token has a loss: no product is empty)
    const int up = max((all + a.unit - 1) / a.unit, 1) * a.unit;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *a.count = up;
        if (a.scale != nullptr) *a.scale = most;
    }
    const int last = min(first + a.per, a.padded), chunks = a.hp / 8;
    for (int t0 = first; t0 < last; t0 += 64) {
        // where the tokens go: those with a loss in their order, the others behind them while there are rows to fill with zeros
        const int t = t0 + lane;
        const bool here = t < last, one = here && t < a.tokens && learned(t);
        const uint64_t mask = __ballot(one);
        const int rank = __popcll(mask & ((1ull << lane) - 1));
        const int dst = one ? before + rank : all + (t0 - before) + (lane - rank);
        const int to = here && dst < up ? dst : -1;
        if (wave == 0) {
            if (to >= 0) {
                a.rows[to] = one ? t : -1;
                a.label32[to] = one ? (int)a.labels[t] : -1;
                if (a.lse != nullptr) {
                    a.lse[to] = one ? a.lse_in[t] : 0.f;
                    a.dloss[to] = one ? a.dloss_in[t] / most : 0.f;
                }
            }
            if (a.loss_out != nullptr && here && t < a.tokens && !one) {
                a.loss_out[t] = 0.f;
                a.lse_out[t] = 0.f;
            }
        }
        const int n = min(64, last - t0);
        for (int r = wave; r < n; r += 4) {              // a row per wave, four chunks of a lane at a time
            const int row = __builtin_amdgcn_readlane(to, r);
            const bool copy = (mask >> r) & 1;
            const uint16_t* src = a.x + (int64_t)(t0 + r) * a.ld;
            uint16_t* zero = !copy && a.dx != nullptr && t0 + r < a.tokens ? a.dx + (int64_t)(t0 + r) * a.ld : nullptr;
            if (row < 0 && zero == nullptr) continue;
            for (int c0 = lane; c0 < chunks; c0 += 256) {
                float v[4][8] = {};
                if (copy)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (c0 + 64 * i < chunks) load_run(src + (c0 + 64 * i) * 8, a.h - (c0 + 64 * i) * 8, v[i]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = (c0 + 64 * i) * 8;
                    if (c >= a.hp) break;
                    if (row >= 0) store_run(a.xc + (int64_t)row * a.hp + c, 8, v[i]);
                    if (zero != nullptr) store_run(zero + c, a.h - c, v[i]);
                }
            }
        }
        before += __popcll(mask);
    }
}

// dl of the entries from v0 on.  4096 tokens, 4096 x 16128: 484 us (1118 TFLOP/s).
struct DLogitsRun {
    static constexpr bool kPair = false, kCounted = true;
    const int32_t* label32;
    const float *lse, *dloss;
    uint16_t* dl;
    int64_t ldc;
    int v0;
    __device__ void split(int) {}
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&v)[R]) const {
        const int label = label32[row];
        const float ref = lse[row] * kLog2e, g = dloss[row];
        const int at = label - v0 - col;
#pragma unroll
        for (int e = 0; e < R; ++e) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[e], kLog2e, -ref)) - (at == e ? 1.f : 0.f);
            v[e] = label >= 0 ? g * p : 0.f;
        }
        store_run(dl + (int64_t)row * ldc + col, left, v);
    }
};

// dx over the pieces and the parts of a split contraction: in fp32 up to the last one, which rounds.  4096 tokens, 16128 x 4096: 462 us
// (1171 TFLOP/s); 512 tokens with a loss, 32003 x 2048 in eight parts 92 us and 9 for their sum, in 64 x 64 tiles that take
// all of it 224.
struct AddRun {
    static constexpr bool kPair = false, kCounted = true;
    float* sum;              // [splits][padded tokens][ld_sum]
    uint16_t* out;
    const int32_t* rows;
    const float* scale;
    int64_t ld_sum, ld_out, stride;
    bool begins, ends;       // with this piece; ends only where there is one split
    __device__ void split(int s) { sum += s * stride; }
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&v)[R]) const {
        float* p = sum + (int64_t)row * ld_sum + col;      // rows of whole 16-byte chunks
        if (!begins) {
#pragma unroll
            for (int e = 0; e < R; e += 4)
                if (e < left) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(p + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[e + k] += b[k];
                }
        }
        if (!ends) {
#pragma unroll
            for (int e = 0; e < R; e += 4)
                if (e < left) *reinterpret_cast<f32x4*>(p + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else if (const int to = rows[row]; to >= 0) {
            const float f = *scale;
#pragma unroll
            for (int e = 0; e < R; ++e) v[e] *= f;
            store_run(out + (int64_t)to * ld_out + col, left, v);
        }
    }
};

// ---- sizes ----
static int check_head(int64_t tokens, int64_t h, int64_t vocab, int64_t& ld) {
    constexpr int64_t most = int64_t(1) << 24;
    if (tokens <= 0 || h <= 0 || vocab <= 0 || tokens >= most || vocab >= most || h >= 65536) return QG_ERR_SHAPE;
    // threads of one launch: tiles of dz, rows of x, tiles of dW
    if (tokens * vocab >= (int64_t(1) << 38) || tokens * h >= (int64_t(1) << 34) || vocab * h >= (int64_t(1) << 37)) return QG_ERR_SHAPE;
    if (ld == 0) ld = h;
    if (ld != h && (ld < h || (ld & 15) || ld >= 65536 + 16)) return QG_ERR_SHAPE;
    return QG_OK;
}
// (labels and the numbers per token are read one by one: a shifted view of a longer array will do)
static bool aligned_to(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Tiles of a product of M x N elements: 256 x 256 with a workgroup per CU at least, 128 x 128, or 64 x 64 where those would leave
// CUs idle.  (64 x 64 below 400 or 520 tiles of 128 x 128 is within 2 %, but slower for 256 tokens, 32000 x 768: forward 31.8 us
// against 24.6.)
enum : int { kTile64 = 0, kTile128 = 1, kTile256 = 2 };
static int head_tile(int64_t M, int64_t N) {
    if (M >= 1024 && ((M + 255) / 256) * ((N + 255) / 256) >= 256) return kTile256;
    return ((M + 127) / 128) * ((N + 127) / 128) < 256 ? kTile64 : kTile128;
}
template <int AL, int BL, typename EPI>
static int launch_head(EpiProduct<LinOperand, EPI> p, int tile, hipStream_t st) {
    switch (tile) {
        case kTile256: return launch_epilogue_shape<AL, BL, 2, 256, 64, 4, true, true, 1, 1>(p, st);
        case kTile128: return launch_epilogue_shape<AL, BL, 2, 128, 64, 2, true, true, 1, 1>(p, st);
        default: return launch_epilogue_shape<AL, BL, 1, 64, 64, 2, true, true, 1, 1>(p, st);
    }
}
// waves' rows of the forward product: slots of a token's partial sums
static int64_t head_slots(int64_t tokens, int64_t vocab) {
    const int tile = head_tile(vocab, tokens);
    const int64_t rows = tile == kTile64 ? 32 : 64, per_tile = tile == kTile256 ? 4 : 2;
    return up(vocab, rows * per_tile) / rows;
}

// dx has tokens x h elements and a contraction as long as the vocabulary: where its tiles would leave CUs idle, the contraction of a
// piece is split over workgroups, 1024 of it each at least, up to two workgroups of 128 x 128 (or 64 x 64) tiles per CU.  The device
// knows how many tokens have a loss, and so how many tiles there are: the grid and the workspace have room for twice the parts that
// all tokens would get, and live_chunk decides.  Backward pass, us, parts for two / for four workgroups per CU: 500 tokens, 32003 x
// 2048 268 / 282 (eight: 320), 700, 32000 x 1024 214 / 232, 1000, 32000 x 768 216 / 237, 100, 32000 x 4096 271 / 277, 2048, 50304 x
// 768 620 / 640; but 1500, 32000 x 2048 690 / 679.  1000 tokens of which half have a loss, 32003 x 2048: two workgroups per CU for the
// tiles that there are 279, for those of all tokens 310.
static int head_dx_tile(int64_t tokens, int64_t h) {
    const int tile = head_tile(tokens, h);
    return tile == kTile64 && tokens > 64 && h > 64 ? kTile128 : tile;
}
static int64_t head_chunk(int64_t tokens, int64_t h, int64_t piece) {
    const int tile = head_dx_tile(tokens, h);
    if (tile == kTile256) return piece;
    const int64_t side = tile == kTile64 ? 64 : 128, tiles = ((tokens + side - 1) / side) * ((h + side - 1) / side);
    const int64_t room = 1024 / tiles, most = piece / 1024, splits = room < most ? room : most;
    return splits <= 1 ? piece : up((piece + splits - 1) / splits, 64);
}

// Entries of a piece: dl of one piece, of all rows that the tokens are padded to, takes 128 MiB at most (so that both products find it in
// the 256 MB cache behind the L2s), but 1024 entries at least (beyond 65536 tokens that is more); pieces of about one size, multiples of
// 256.  4096 tokens, us, pieces of 128 / 64 MiB: 32000 x 768 1002 / 1171, 32000 x 4096 3895 / 4006.
static int64_t head_piece(int64_t padded, int64_t vocab) {
    const int64_t most = (int64_t(1) << 26) / padded / 256 * 256;
    const int64_t piece = most < 1024 ? 1024 : most;
    const int64_t pieces = (vocab + piece - 1) / piece;
    const int64_t even = up((vocab + pieces - 1) / pieces, 256);
    return even < vocab ? even : vocab;
}

struct HeadSpace {     // a call's workspace, in bytes
    int64_t piece, chunk, splits, hp, unit, padded, slots;     // chunk: least contraction of dx per workgroup; splits: most parts
    size_t count, scale, rows, labels, lse, dloss, x, sum, dl, part, logit, total;
};
static HeadSpace head_space(int64_t tokens, int64_t h, int64_t vocab, bool backward) {
    HeadSpace s = {};
    s.hp = up(h, backward ? 256 : 8);
    // whole rows of the largest tile that the products may take (32 tokens, 32000 x 768, backward: 54 us, 87 with 256 throughout)
    s.unit = tokens <= 64 ? 64 : tokens <= 512 ? 128 : 256;
    s.padded = up(tokens, s.unit);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    s.count = take(4);
    s.scale = take(4);
    s.rows = take((size_t)s.padded * 4);
    s.labels = take((size_t)s.padded * 4);
    s.x = take((size_t)s.padded * s.hp * 2);
    if (backward) {
        s.piece = head_piece(s.padded, vocab);
        s.chunk = head_chunk(s.padded, h, s.piece);
        s.splits = (s.piece + s.chunk - 1) / s.chunk;
        s.lse = take((size_t)s.padded * 4);
        s.dloss = take((size_t)s.padded * 4);
        s.sum = take(s.piece < vocab || s.splits > 1 ? (size_t)s.padded * s.hp * 4 * s.splits : 0);
        s.dl = take((size_t)s.padded * up(s.piece, kLinTM) * 2);
    } else {
        s.slots = head_slots(s.padded, vocab);
        s.part = take((size_t)s.padded * 8 * s.slots);
        s.logit = take((size_t)s.padded * 4);
    }
    s.total = at;
    return s;
}

// Whether the forward pass puts the tokens that have a loss together: it costs one launch and a copy of x, 6 us and more, which
// a product of 2^36 flop (some 80 us) or more is worth; the backward pass, of three products, always does.
static bool head_put_together(int64_t tokens, int64_t h, int64_t vocab) { return 2. * tokens * h * vocab >= 68719476736.; }

static int launch_head_rows(HeadRows a, hipStream_t st) {
    // a token per wave, or as many as make a thousand workgroups (each counts all labels)
    const int64_t per = (a.padded + 1023) / 1024;
    a.per = (int)(per < 4 ? 4 : per);
    hipLaunchKernelGGL(k_head_rows, dim3((unsigned)((a.padded + a.per - 1) / a.per)), dim3(256), 0, st, a);
    return check_launch();
}

// dW's rows of a piece, dl^T x: direct loads of whole tiles (4096 tokens, 16128 x 4096: 488 us, 1109 TFLOP/s; 512, 32003 x 2048: 87 to 95,
// through registers 113).  dl's rows are a multiple of 128 elements apart, x's of 256, so that a
// tile never leaves its row; what stands between their ends and that only reaches elements that are not stored.  (The sizes' limits keep
// both below kKSlowPitch.)
static int launch_head_dw(const uint16_t* dl, int64_t pitch, const uint16_t* x, int64_t hp, uint16_t* dW, int64_t ldc, int64_t width,
                          int64_t h, int64_t padded, const int32_t* count, const float* scale, hipStream_t st) {
    const int64_t tiles_m = pitch / kLinTM, tiles_n = hp / 256;
    const KSlowOut out = {(int)width, (int)h, ldc, count, nullptr, nullptr, scale};
    hipLaunchKernelGGL((k_gemm_kslow_direct<uint16_t, true>), dim3((unsigned)((tiles_m * tiles_n + 7) / 8 * 8)), dim3(256), 0, st, dl, x, dW,
                       (int)pitch, (int)hp, (int)padded, (int)tiles_m, (int)tiles_n, out);
    return check_launch();
}

}  // namespace qg

using namespace qg;

extern "C" size_t qg_head_loss_workspace_bytes(int64_t tokens, int64_t h, int64_t vocab) {
    int64_t ld = 0;
    if (check_head(tokens, h, vocab, ld)) return 0;
    const size_t f = head_space(tokens, h, vocab, false).total, b = head_space(tokens, h, vocab, true).total;
    return f > b ? f : b;
}

extern "C" int qg_head_loss_forward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, int64_t tokens, int64_t h,
                                    int64_t vocab, int64_t ld, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    if (!x_bf16 || !W_bf16 || !labels || !loss || !lse) return QG_ERR_NULL;
    if (int e = check_head(tokens, h, vocab, ld)) return e;
    if (!aligned16(x_bf16) || !aligned16(W_bf16) || !aligned16(workspace) || !aligned_to(labels, 8) || !aligned_to(loss, 4) ||
        !aligned_to(lse, 4))
        return QG_ERR_ALIGN;
    const HeadSpace s = head_space(tokens, h, vocab, false);
    if (!workspace || workspace_bytes < s.total) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    char* at = static_cast<char*>(workspace);
    HeadRows r = {};
    EpiProduct<LinOperand, StatsEpilogue> p;
    p.A = p.A2 = LinOperand{W_bf16, nullptr, ld, 0};
    p.B = p.B2 = LinOperand{x_bf16, nullptr, ld, 0};
    p.M = (int)vocab, p.N = (int)tokens, p.K = (int)h;
    if (head_put_together(tokens, h, vocab)) {
        r.x = x_bf16, r.labels = labels, r.ld = ld, r.vocab = vocab;
        r.tokens = (int)tokens, r.padded = (int)s.padded, r.unit = (int)s.unit, r.h = (int)h, r.hp = (int)s.hp;
        r.xc = reinterpret_cast<uint16_t*>(at + s.x);
        r.rows = reinterpret_cast<int32_t*>(at + s.rows);
        r.label32 = reinterpret_cast<int32_t*>(at + s.labels);
        r.count = reinterpret_cast<int32_t*>(at + s.count);
        r.loss_out = loss, r.lse_out = lse;
        if (int e = launch_head_rows(r, st)) return e;
        p.B = p.B2 = LinOperand{r.xc, nullptr, s.hp, 0};
        p.N = (int)s.padded;
        p.count = r.count;
        p.dim = kDimN;
        p.unit = (int)s.unit;
    }
    f32x2* part = reinterpret_cast<f32x2*>(at + s.part);
    float* label_logit = reinterpret_cast<float*>(at + s.logit);
    p.epi = StatsEpilogue{r.label32, labels, label_logit, part, s.padded};
    if (int e = launch_head<kBf16KFast, kBf16KFast>(p, head_tile(vocab, s.padded), st)) return e;
    hipLaunchKernelGGL(k_head_join, dim3((unsigned)((s.padded + 15) / 16)), dim3(1024), 0, st, part, (int)s.slots, s.padded, labels, vocab,
                       r.rows, label_logit, r.count, p.N, loss, lse);
    return check_launch();
}

extern "C" int qg_head_loss_backward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, const float* lse,
                                     const float* dloss, int64_t tokens, int64_t h, int64_t vocab, int64_t ld, uint16_t* dx_bf16,
                                     uint16_t* dW_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x_bf16 || !W_bf16 || !labels || !lse || !dloss || (!dx_bf16 && !dW_bf16)) return QG_ERR_NULL;
    if (int e = check_head(tokens, h, vocab, ld)) return e;
    if (!aligned16(x_bf16) || !aligned16(W_bf16) || !aligned16(dx_bf16) || !aligned16(dW_bf16) || !aligned16(workspace) ||
        !aligned_to(labels, 8) || !aligned_to(lse, 4) || !aligned_to(dloss, 4))
        return QG_ERR_ALIGN;
    const HeadSpace s = head_space(tokens, h, vocab, true);
    if (!workspace || workspace_bytes < s.total) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    char* at = static_cast<char*>(workspace);
    HeadRows r = {};
    r.x = x_bf16, r.labels = labels, r.lse_in = lse, r.dloss_in = dloss, r.ld = ld, r.vocab = vocab;
    r.tokens = (int)tokens, r.padded = (int)s.padded, r.unit = (int)s.unit, r.h = (int)h, r.hp = (int)s.hp;
    r.xc = reinterpret_cast<uint16_t*>(at + s.x);
    r.rows = reinterpret_cast<int32_t*>(at + s.rows);
    r.label32 = reinterpret_cast<int32_t*>(at + s.labels);
    r.count = reinterpret_cast<int32_t*>(at + s.count);
    r.lse = reinterpret_cast<float*>(at + s.lse);
    r.dloss = reinterpret_cast<float*>(at + s.dloss);
    r.scale = reinterpret_cast<float*>(at + s.scale);
    r.dx = dx_bf16;
    if (int e = launch_head_rows(r, st)) return e;
    uint16_t* dl = reinterpret_cast<uint16_t*>(at + s.dl);
    float* sum = reinterpret_cast<float*>(at + s.sum);
    const int64_t stride = s.padded * s.hp;
    LiveParts live;
    live.k = (int)s.piece, live.chunk = (int)s.chunk;
    live.side = head_dx_tile(s.padded, h) == kTile64 ? 64 : 128;
    live.across = (int)((h + live.side - 1) / live.side);
    for (int64_t v0 = 0; v0 < vocab; v0 += s.piece) {
        const int64_t width = vocab - v0 < s.piece ? vocab - v0 : s.piece, pitch = up(width, kLinTM);
        const LinOperand x = {r.xc, nullptr, s.hp, 0}, W = {W_bf16 + v0 * ld, nullptr, ld, 0}, d = {dl, nullptr, pitch, 0};
        {
            EpiProduct<LinOperand, RunEpilogue<DLogitsRun>> p;
            p.A = p.A2 = x;
            p.B = p.B2 = W;
            static_cast<DLogitsRun&>(p.epi) = DLogitsRun{r.label32, r.lse, r.dloss, dl, pitch, (int)v0};
            p.M = (int)s.padded, p.N = (int)width, p.K = (int)h;
            p.count = r.count;
            p.dim = kDimM;
            p.unit = (int)s.unit;
            if (int e = launch_head<kBf16KFast, kBf16KFast>(p, head_tile(s.padded, width), st)) return e;
        }
        if (dx_bf16) {
            EpiProduct<LinOperand, RunEpilogue<AddRun>> p;
            p.A = p.A2 = d;
            p.B = p.B2 = W;
            static_cast<AddRun&>(p.epi) = AddRun{sum, dx_bf16, r.rows, r.scale, s.hp, ld, stride, v0 == 0, v0 + width == vocab && s.splits == 1};
            p.M = (int)s.padded, p.N = (int)h, p.K = (int)width;
            p.count = r.count;
            p.dim = kDimM;
            p.unit = (int)s.unit;
            p.k_chunk = (int)s.chunk;
            p.live_k = live.k;
            p.splits = (int)((width + s.chunk - 1) / s.chunk);
            if (int e = launch_head<kBf16KFast, kBf16KSlow>(p, head_dx_tile(s.padded, h), st)) return e;
        }
        if (dW_bf16)
            if (int e = launch_head_dw(dl, pitch, r.xc, s.hp, dW_bf16 + v0 * ld, ld, width, h, s.padded, r.count, r.scale, st)) return e;
    }
    if (dx_bf16 && s.splits > 1)
        return launch_join_parts(sum, s.hp, stride, (int)s.splits, live, r.rows, r.count, r.scale, s.padded, h, dx_bf16, ld, st);
    return QG_OK;
}
