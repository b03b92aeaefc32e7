// Cross entropy of a language model's head over its vocabulary, without the logits in memory.  With x [T][h], W [V][h],
// z = x W^T:
//     lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,label
//     dl_tv = dloss_t (exp(z_tv - lse_t) - [v = label]),   dx = dl W,   dW = dl^T x
// forward:  one product whose epilogue leaves, of every tile, each token's maximum and sum of exponentials over the tile's
//           entries, and the label's logit; a second kernel joins them.  The product is computed as W x^T, so that a lane's sums
//           belong to one token and most of the reduction stays in its registers.
// backward: the vocabulary in pieces.  For each, the logits are computed again with dl in the epilogue (bf16, the operand of the
//           two products), then dW's rows of the piece, and dx, which is added up over the pieces in fp32.
// Eight T V h flop against six with the logits kept; T x V numbers are never stored, only T x piece.
#include "qg_epilogue.h"

namespace qg {

constexpr float kLog2e = 1.44269504f;

// ---- forward ----
// Rows of the product are vocabulary entries, columns tokens.  A lane has 16 entries of each block of its column's token, the lane 32
// further the other 16.
struct StatsEpilogue {
    static constexpr bool kPair = false;
    const int64_t* labels;
    float* label_logit;
    f32x2* part;        // [slots][N]: maximum and sum of exp(z - maximum) over a wave's 32 MB rows
    template <bool EXACT, int MB, int NB>
    __device__ __forceinline__ void tile(const f32x16 (&acc)[MB][NB], float*, int row0, int col0, bool inside, int M, int N,
                                         int lane) const {
        const int slot = row0 / (32 * MB), sub = 4 * (lane >> 5);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int col = col0 + b * 32 + (lane & 31);
            const bool token = EXACT || inside || col < N;
            const int64_t label = token ? labels[col] : -1;
            const int at = label >= 0 && label < M ? (int)label - row0 - sub : -1;     // row of the label among the lane's
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
            if (lane < 32 && token) part[(int64_t)slot * N + col] = f32x2{top, sum};
        }
    }
};

__device__ __forceinline__ void join(float& top, float& sum, float top2, float sum2) {
    const float t = fmaxf(top, top2);
    const float ref = t == -INFINITY ? 0.f : t;
    sum = sum * __builtin_amdgcn_exp2f((top - ref) * kLog2e) + sum2 * __builtin_amdgcn_exp2f((top2 - ref) * kLog2e);
    top = t;
}

// 16 tokens per workgroup, 64 slices of the slots, joined in a fixed order.
__global__ __launch_bounds__(1024) void k_head_join(const f32x2* __restrict__ part, int slots, const int64_t* __restrict__ labels,
                                                    const float* __restrict__ label_logit, int tokens, int64_t vocab,
                                                    float* __restrict__ loss, float* __restrict__ lse) {
    __shared__ float tops[64][17], sums[64][17];
    const int lane = threadIdx.x & 15, slice = threadIdx.x >> 4, t = blockIdx.x * 16 + lane;
    float top = -INFINITY, sum = 0.f;
    if (t < tokens)
        for (int s = slice; s < slots; s += 64) {
            const f32x2 p = part[(int64_t)s * tokens + t];
            join(top, sum, p[0], p[1]);
        }
    tops[slice][lane] = top;
    sums[slice][lane] = sum;
#pragma unroll
    for (int n = 32; n > 0; n >>= 1) {
        __syncthreads();
        if (slice < n) {
            join(top, sum, tops[slice + n][lane], sums[slice + n][lane]);
            tops[slice][lane] = top;
            sums[slice][lane] = sum;
        }
    }
    if (slice != 0 || t >= tokens) return;
    const float l = top + logf(sum);
    const int64_t label = labels[t];
    lse[t] = l;
    loss[t] = label >= 0 && label < vocab ? l - label_logit[t] : 0.f;
}

// ---- backward ----
// x with zeros where a token has no loss (0 times what stands there would be NaN in dW if that is not finite), rows padded to whole
// 16-byte chunks; and each token's label in 32 bits, -1 for none.
__global__ __launch_bounds__(256) void k_head_rows(const uint16_t* __restrict__ x, const int64_t* __restrict__ labels, int tokens, int h,
                                                   int64_t ld, int hp, int64_t vocab, uint16_t* __restrict__ xm, int32_t* __restrict__ label32) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = hp / 8;
    const int64_t t = i / per;
    if (t >= tokens) return;
    const int col = (int)(i - t * per) * 8;
    const int64_t label = labels[t];
    const bool learned = label >= 0 && label < vocab;
    float v[8] = {};
    if (learned) load_run(x + t * ld + col, h - col, v);
    store_run(xm + t * hp + col, 8, v);
    if (col == 0) label32[t] = learned ? (int)label : -1;
}

// dl of the entries from v0 on
struct DLogitsRun {
    static constexpr bool kPair = false;
    const int32_t* label32;
    const float *lse, *dloss;
    uint16_t* dl;
    int64_t ldc;
    int v0;
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

// dx over the pieces: in fp32 up to the last one, which rounds.
struct AddRun {
    static constexpr bool kPair = false;
    const float* before;     // NULL: the first piece
    float* sum;              // NULL: the last piece
    uint16_t* out;
    int64_t ld_sum, ld_out;
    template <int R>
    __device__ __forceinline__ void run(int row, int col, int left, float (&v)[R]) const {
        const int64_t at = (int64_t)row * ld_sum + col;      // rows of whole 16-byte chunks
        if (before != nullptr) {
#pragma unroll
            for (int e = 0; e < R; e += 4)
                if (e < left) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(before + at + e);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[e + k] += b[k];
                }
        }
        if (sum != nullptr) {
#pragma unroll
            for (int e = 0; e < R; e += 4)
                if (e < left) *reinterpret_cast<f32x4*>(sum + at + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
            store_run(out + (int64_t)row * ld_out + col, left, v);
        }
    }
};

// ---- sizes ----
static int check_head(int64_t tokens, int64_t h, int64_t vocab, int64_t& ld) {
    constexpr int64_t most = int64_t(1) << 24;
    if (tokens <= 0 || h <= 0 || vocab <= 0 || tokens >= most || vocab >= most || h >= 65536) return QG_ERR_SHAPE;
    if (tokens * vocab >= (int64_t(1) << 38) || tokens * h >= (int64_t(1) << 34)) return QG_ERR_SHAPE;   // threads of one launch
    if (ld == 0) ld = h;
    if (ld != h && (ld < h || (ld & 15) || ld >= 65536 + 16)) return QG_ERR_SHAPE;
    return QG_OK;
}
static int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Tiles of a product of M x N elements: 256 x 256 with a workgroup per CU at least, 128 x 128, or 64 x 64 where those would leave
// half of the CUs idle.
enum : int { kTile64 = 0, kTile128 = 1, kTile256 = 2 };
static int head_tile(int64_t M, int64_t N) {
    if (M >= 1024 && ((M + 255) / 256) * ((N + 255) / 256) >= 256) return kTile256;
    return ((M + 127) / 128) * ((N + 127) / 128) < 256 ? kTile64 : kTile128;
}
template <int AL, int BL, typename EPI>
static int launch_head(EpiProduct<LinOperand, EPI> p, hipStream_t st) {
    switch (head_tile(p.M, p.N)) {
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

// Entries of a piece: dl of one piece stays below 64 MiB (so that both products find it in the 256 MB cache behind the L2s), 1024
// entries at least, pieces of about one size.
static int64_t head_piece(int64_t tokens, int64_t vocab) {
    const int64_t most = (int64_t(1) << 25) / tokens;
    const int64_t piece = most < 1024 ? 1024 : most;
    const int64_t pieces = (vocab + piece - 1) / piece;
    const int64_t even = up((vocab + pieces - 1) / pieces, 256);
    return even < vocab ? even : vocab;
}

struct HeadSpace {     // the backward pass's workspace, in bytes
    int64_t piece, hp;
    size_t labels, x, sum, dl, total;
};
static HeadSpace head_space(int64_t tokens, int64_t h, int64_t vocab) {
    HeadSpace s;
    s.piece = head_piece(tokens, vocab);
    s.hp = up(h, 8);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    s.labels = take((size_t)tokens * 4);
    s.x = take((size_t)tokens * s.hp * 2);
    s.sum = take(s.piece < vocab ? (size_t)tokens * s.hp * 4 : 0);
    s.dl = take((size_t)tokens * up(s.piece, 16) * 2);
    s.total = at;
    return s;
}
static size_t head_forward_bytes(int64_t tokens, int64_t vocab) {
    return (size_t)tokens * 8 * head_slots(tokens, vocab) + (size_t)up(tokens, 4) * 4;
}

}  // namespace qg

using namespace qg;

extern "C" size_t qg_head_loss_workspace_bytes(int64_t tokens, int64_t h, int64_t vocab) {
    int64_t ld = 0;
    if (check_head(tokens, h, vocab, ld)) return 0;
    const size_t f = head_forward_bytes(tokens, vocab), b = head_space(tokens, h, vocab).total;
    return f > b ? f : b;
}

extern "C" int qg_head_loss_forward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, int64_t tokens, int64_t h,
                                    int64_t vocab, int64_t ld, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                                    void* stream) {
    if (!x_bf16 || !W_bf16 || !labels || !loss || !lse) return QG_ERR_NULL;
    if (int e = check_head(tokens, h, vocab, ld)) return e;
    for (const void* p : {(const void*)x_bf16, (const void*)W_bf16, (const void*)labels, (const void*)loss, (const void*)lse,
                          (const void*)workspace})
        if (!aligned16(p)) return QG_ERR_ALIGN;
    if (!workspace || workspace_bytes < head_forward_bytes(tokens, vocab)) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t slots = head_slots(tokens, vocab);
    f32x2* part = static_cast<f32x2*>(workspace);
    float* label_logit = reinterpret_cast<float*>(part + slots * tokens);
    EpiProduct<LinOperand, StatsEpilogue> p;
    p.A = p.A2 = LinOperand{W_bf16, nullptr, ld, 0};
    p.B = p.B2 = LinOperand{x_bf16, nullptr, ld, 0};
    p.epi = StatsEpilogue{labels, label_logit, part};
    p.M = (int)vocab, p.N = (int)tokens, p.K = (int)h;
    if (int e = launch_head<kBf16KFast, kBf16KFast>(p, st)) return e;
    hipLaunchKernelGGL(k_head_join, dim3((unsigned)((tokens + 15) / 16)), dim3(1024), 0, st, part, (int)slots, labels, label_logit,
                       (int)tokens, vocab, loss, lse);
    return check_launch();
}

extern "C" int qg_head_loss_backward(const uint16_t* x_bf16, const uint16_t* W_bf16, const int64_t* labels, const float* lse,
                                     const float* dloss, int64_t tokens, int64_t h, int64_t vocab, int64_t ld, uint16_t* dx_bf16,
                                     uint16_t* dW_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    if (!x_bf16 || !W_bf16 || !labels || !lse || !dloss || (!dx_bf16 && !dW_bf16)) return QG_ERR_NULL;
    if (int e = check_head(tokens, h, vocab, ld)) return e;
    for (const void* p : {(const void*)x_bf16, (const void*)W_bf16, (const void*)labels, (const void*)lse, (const void*)dloss,
                          (const void*)dx_bf16, (const void*)dW_bf16, (const void*)workspace})
        if (!aligned16(p)) return QG_ERR_ALIGN;
    const HeadSpace s = head_space(tokens, h, vocab);
    if (!workspace || workspace_bytes < s.total) return QG_ERR_WORKSPACE;
    const hipStream_t st = (hipStream_t)stream;
    char* at = static_cast<char*>(workspace);
    int32_t* label32 = reinterpret_cast<int32_t*>(at + s.labels);
    uint16_t *xm = reinterpret_cast<uint16_t*>(at + s.x), *dl = reinterpret_cast<uint16_t*>(at + s.dl);
    float* sum = reinterpret_cast<float*>(at + s.sum);
    hipLaunchKernelGGL(k_head_rows, dim3((unsigned)((tokens * (s.hp / 8) + 255) / 256)), dim3(256), 0, st, x_bf16, labels, (int)tokens,
                       (int)h, ld, (int)s.hp, vocab, xm, label32);
    if (int e = check_launch()) return e;
    for (int64_t v0 = 0; v0 < vocab; v0 += s.piece) {
        const int64_t width = vocab - v0 < s.piece ? vocab - v0 : s.piece, pitch = up(width, 16);
        const LinOperand x = {xm, nullptr, s.hp, 0}, W = {W_bf16 + v0 * ld, nullptr, ld, 0}, d = {dl, nullptr, pitch, 0};
        {
            EpiProduct<LinOperand, RunEpilogue<DLogitsRun>> p;
            p.A = p.A2 = x;
            p.B = p.B2 = W;
            static_cast<DLogitsRun&>(p.epi) = DLogitsRun{label32, lse, dloss, dl, pitch, (int)v0};
            p.M = (int)tokens, p.N = (int)width, p.K = (int)h;
            if (int e = launch_head<kBf16KFast, kBf16KFast>(p, st)) return e;
        }
        if (dx_bf16) {
            EpiProduct<LinOperand, RunEpilogue<AddRun>> p;
            p.A = p.A2 = d;
            p.B = p.B2 = W;
            const bool last = v0 + width == vocab;
            static_cast<AddRun&>(p.epi) = AddRun{v0 > 0 ? sum : nullptr, last ? nullptr : sum, dx_bf16, s.hp, ld};
            p.M = (int)tokens, p.N = (int)h, p.K = (int)width;
            if (int e = launch_head<kBf16KFast, kBf16KSlow>(p, st)) return e;
        }
        if (dW_bf16)
            if (int e = launch_tile_gemm<kBf16KSlow, kBf16KSlow, uint16_t>(d, x, nullptr, dW_bf16 + v0 * ld, width, h, tokens, st, nullptr,
                                                                           1, ld))
                return e;
    }
    return QG_OK;
}
