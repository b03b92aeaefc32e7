// What the attention kernels share: the geometry of packed sequences, tiles of keys or queries in LDS, scores and masks.
//
// Tokens are packed: sequence i has queries cu_q[i] .. cu_q[i + 1] - 1 and keys cu_k[i] .. cu_k[i + 1] - 1, and its queries are the last of
// its keys: query i stands at position p = i + n_k - n_q.  For a query, the visible keys are an interval lo <= j <= hi:
//     hi = n_k - 1, causal: min(that, max(p, prefix - 1));     lo = 0, with a window: p - window + 1
// both growing with p, so that whole tiles are seen by all rows, by none, or need a test per score.
//
// Operand layouts (v_mfma_f32_32x32x16_bf16): an operand's lane l holds row or column l % 32 and 8 values of k; the accumulator's
// register v of lane l is [8 (v / 4) + 4 (l / 32) + v % 4][l % 32].  Scores are computed with the index that the next product sums over as
// their row: a lane then holds, for one column, the values of k that the next product wants in one operand, in an order of k of its own
// (first 4 h .. 4 h + 3, then 8 + 4 h .. 8 + 4 h + 3 of each 16, h = l / 32), and the other operand is read in that order.
// So probabilities never leave the registers.
#pragma once
#include "qg_common.h"
#include "qg_gemm_kernels.h"

namespace qg {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

constexpr int64_t kAttnMaxTokens = int64_t(1) << 24;
constexpr int kAttnMaxHeads = 1024, kAttnMaxSequences = 1 << 20;
constexpr int64_t kHeadsMaxStride = int64_t(1) << 23;   // elements between tokens: 128 rows are addressed in 31 bits from one base

int check_heads(const qg_heads* x, bool required, int unit = 8);    // host, qg_attention.hip; unit: elements that address and strides are multiples of
int check_cache(const qg_cache* c);                     // host, qg_rope.hip
// Scale and cap such that their quotient, and its products with a score, are numbers of fp32 (a cap of 10^-40 made a score of 0 NaN).
inline bool check_scores(float scale, float cap) {
    return scale >= 0x1p-60f && scale <= 0x1p60f && (cap == 0.f || (cap >= 0x1p-60f && cap <= 0x1p60f));
}

struct AttnArgs {
    int64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, o_ts, o_hs, do_ts, do_hs, dq_ts, dq_hs, dk_ts, dk_hs, dv_ts, dv_hs;   // strides, elements
    const uint16_t *q, *k, *v, *dO;
    uint16_t *o, *dq, *dk, *dv;
    float* lse;          // [heads_q][tokens_q]
    float* stats;        // [2][heads_q][tokens_q]: what dkv begins the products at
    const int32_t *cu_q, *cu_k, *prefix;
    const float* slopes;
    float* part;         // sums of parts, to be joined (see qg_attention.hip)
    int tokens_q, tokens_k, heads_q, group, d, sequences, causal, window, tiles, parts;
    float scale, cap;
};

// One tile of a sequence's rows.
struct AttnTile {
    int seq;       // `sequences`: the rows behind the last sequence
    int tile;      // of the sequence
    int q0, nq, k0, nk, prefix;
};

// Boundary i of packed sequences, inside the tokens whatever memory holds.
__device__ __forceinline__ int attn_boundary(const int32_t* cu, int i, int sequences, int tokens) {
    int at = tokens;
    if (cu != nullptr) at = cu[min(i, sequences)];
    return i == 0 ? 0 : min(max(at, 0), tokens);
}

// Tile t of the rows in blocks of BM per sequence.  Sequence i's tiles are numbered from boundary_i / BM + i on: that leaves room for each
// sequence's last, partial one without a sum over the sequences before it (a number too many has no rows).  The rows behind the
// last sequence are one more.  63 boundaries are looked at at once, and the next; the first always counts, so each turn narrows the range.  The last
// turn's lanes hold the sequence's own boundaries.  (Loading them again, and rows by loads with a branch each: 16 sequences of 256 tokens, 16 heads of 64,
// forward 13.2 -> 13.6 us, backward 39.6 -> 42.4.)
// KEYS: the rows are keys.  The rows behind the last sequence have no partners.
// Boundaries that descend can give a tile ahead of its sequence, of a negative number: it has no rows (as rows they would be those of other sequences).
template <int BM, bool KEYS>
__device__ __forceinline__ AttnTile attn_tile(const AttnArgs& a, int t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.sequences + 1, step, count, q, k;
    do {
        step = (n + 62) / 63;
        const int at = lane * step;
        q = attn_boundary(a.cu_q, lo + at, a.sequences, a.tokens_q);
        k = attn_boundary(a.cu_k, lo + at, a.sequences, a.tokens_k);
        count = min(63, max(1, (int)__popcll(__ballot(at < n && (KEYS ? k : q) / BM + lo + at <= t))));
        lo += (count - 1) * step;
        n = min(step, n - (count - 1) * step);
    } while (step > 1);
    AttnTile r;
    r.seq = lo;
    r.q0 = __builtin_amdgcn_readlane(q, count - 1);
    r.k0 = __builtin_amdgcn_readlane(k, count - 1);
    r.tile = t - ((KEYS ? r.k0 : r.q0) / BM + lo);
    const bool tail = lo >= a.sequences;
    const int q1 = tail ? a.tokens_q : __builtin_amdgcn_readlane(q, count);
    const int k1 = tail ? a.tokens_k : __builtin_amdgcn_readlane(k, count);
    r.nq = tail && KEYS ? 0 : max(0, q1 - r.q0);
    r.nk = tail && !KEYS ? 0 : max(0, k1 - r.k0);
    r.prefix = a.prefix != nullptr && !tail ? max(0, a.prefix[lo]) : 0;
    return r;
}

// Workgroup id -> (head, tile of rows, part of what passes by).  Workgroups go to the 8 XCDs in turn; each XCD gets consecutive tiles of
// consecutive heads, so that the keys and values of a head are read into one L2.
__device__ __forceinline__ bool attn_place(int heads, int tiles, int parts, int& head, int& tile, int& part) {
    const int work = heads * tiles * parts, per = (work + 7) / 8, at = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (at >= work) return false;
    const int rest = at / parts;
    part = at - rest * parts;
    head = rest / tiles;
    tile = rest - head * tiles;
    return true;
}

// Steps begin .. end - 1 of `all` that belong to a part.
__device__ __forceinline__ void attn_share(int all, int parts, int part, int& begin, int& end) {
    const int per = all / parts, more = all - per * parts;
    begin = per * part + min(part, more);
    end = begin + per + (part < more ? 1 : 0);
}

// Rows of a [rows][d] bf16 array as an LDS tile of `ROWS` rows of pitch P (64 or 128 elements), by direct loads.  The 16-byte chunk c of row r
// is kept in slot c ^ swizzle(r): reads of one chunk of 16 consecutive rows (an operand whose k is d), transposing reads of four
// chunks of four consecutive rows (an operand whose k is the row) and of two chunks of eight each take every bank once.  All 64 banks are one row at
// P = 128 and two at P = 64, so that there the row's lowest bit places it already.  (P = 64 swizzled by that bit too: each
// read took twice as long, 8192 tokens, 32 heads of 64, backward 1161 -> 1149 us.)
// Rows from `valid` on and elements from d on become zero.
template <int P>
__device__ __forceinline__ int tile_swizzle(int r) {
    return (P == 128 ? (r & 3) << 2 : (r & 2) << 1) | ((r >> 1) & 2) | ((r >> 3) & 1);
}

template <int P, int ROWS, int NT>
struct RowsTile {
    static constexpr int CPR = P / 8, PER = ROWS * CPR / NT, STEP = NT / CPR;   // chunks per row, loads per thread, rows per load
    static_assert(STEP % 16 == 0, "a thread's rows share their swizzle");
    uint32_t off;      // of the thread's first chunk, from the tile's first row
    int row;
    bool in;           // the chunk lies below d
    __device__ __forceinline__ void init(int64_t stride, int d) {
        const int idx = threadIdx.x;
        row = idx / CPR;
        const int chunk = (idx % CPR) ^ tile_swizzle<P>(row);
        in = chunk * 8 < d;
        off = (uint32_t)(row * (int)stride + chunk * 8) * 2u;
    }
    // lds: the tile; rows from `base` on, `valid` of them (more than ROWS: all)
    __device__ __forceinline__ void load(uint16_t* lds, const uint16_t* base, int64_t stride, int valid) const {
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(base);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            const bool there = in && row + p * STEP < valid;
            buffer_load_lds16(rs, lds + p * NT * 8 + wave * 512, there ? off + (uint32_t)(p * STEP) * (uint32_t)stride * 2u : 0x80000000u, 0);
        }
    }
};

// Address in LDS of a tile, a multiple of its rows' pitch.
__device__ __forceinline__ uint32_t tile_address(const uint16_t* tile) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint16_t*)tile;
}
// Reads of a tile's operands.  A lane's address is one number per tile: steps and blocks change the slot alone, by exclusive or, and rows are
// constant offsets.  (Separate addresses for each step and block were 24 registers, of 256 that spill.)
// Reads from LDS that the compiler takes for reads of what no direct load in flight writes: each step waits for its own tile.  (Without `__restrict__`
// it waits for every such load ahead of a transposing read, so for the next step's rows in the middle of this one.)
__device__ __forceinline__ s16x4 lds_read_tr(lds_s16x4* __restrict__ p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p); }
typedef __attribute__((address_space(3))) const f32x4 lds_f32x4;
__device__ __forceinline__ f32x4 lds_read4(lds_f32x4* __restrict__ p) { return *p; }

template <int P>
struct TileReader {
    uint32_t rows, columns;
    __device__ __forceinline__ explicit TileReader(int lane) {
        const int r = lane & 31, s = lane & 15, g = lane >> 4, t = 4 * (g >> 1) + (s >> 2);
        rows = r * P * 2 + ((lane >> 5) ^ tile_swizzle<P>(r)) * 16;
        columns = t * P * 2 + ((2 * (g & 1) + ((s & 3) >> 1)) ^ tile_swizzle<P>(t)) * 16 + 8 * (s & 1);
    }
    // Operand of 32 rows (from row0 on) with k = d, 16 elements from 16 * step on; at: the tile's address + rows.
    __device__ __forceinline__ static bf16x8 frag(uint32_t at, int row0, int step) {
        return *(__attribute__((address_space(3))) const bf16x8*)((at ^ (uint32_t)(step * 32)) + (uint32_t)(row0 * P * 2));
    }
    // Operand of 32 elements of d (from 32 * block on) with k = 16 rows from row0 on, in the order of k of a score's registers; at: the tile's
    // address + columns.
    __device__ __forceinline__ static bf16x8 frag_t(uint32_t at, int row0, int block) {
        const uint32_t lo = at ^ (uint32_t)(block * 64), hi = at ^ (uint32_t)(block * 64 ^ 16);    // (8 rows on the swizzle differs by 1)
        const s16x4 x = lds_read_tr((lds_s16x4*)(lo + (uint32_t)(row0 * P * 2)));
        const s16x4 y = lds_read_tr((lds_s16x4*)(hi + (uint32_t)((row0 + 8) * P * 2)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// The same k = d operand straight from memory: row 32 * wave + lane % 32 from `base` on, if it is there; elements from d on are zero.  (Buffer loads: no
// branch around each of them.)
struct RowFrags {
    __amdgpu_buffer_rsrc_t rs;
    uint32_t off;
    int d, chunk;
    __device__ __forceinline__ RowFrags(const uint16_t* base, int64_t stride, int wave, int lane, bool there, int width) : rs(make_rsrc(base)) {
        chunk = lane >> 5;
        d = there ? width : 0;
        off = (uint32_t)((32 * wave + (lane & 31)) * (int)stride + chunk * 8) * 2u;
    }
    __device__ __forceinline__ bf16x8 get(int step) const {
        return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, (2 * step + chunk) * 8 < d ? off + 32u * step : 0x80000000u, 0, 0));
    }
};

// use(i, operands) for i = 0 .. N - 1, the operands of i + 1 read from LDS before the products of i begin: with 250 of 256 registers taken the
// compiler reads an operand and waits for it, time after time.  (Two ahead spill: 8192 tokens, 32 heads of 128, dq and dkv 1210 -> 1305 us.)
template <int N, typename OPERANDS, typename READ, typename USE>
__device__ __forceinline__ void read_ahead(READ read, USE use) {
    OPERANDS x[2];
    read(0, x[0]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + 1 < N) read(i + 1, x[(i + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
        use(i, x[i & 1]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Registers 8 t .. 8 t + 7 of a score block as the operand of the next product's step t.  Rounded to bf16, an operand of the matrix unit.
__device__ __forceinline__ bf16x8 score_frag(const f32x16& s, int t) {
    const u32x4 w = {pack_bf16x2(s[8 * t], s[8 * t + 1]), pack_bf16x2(s[8 * t + 2], s[8 * t + 3]), pack_bf16x2(s[8 * t + 4], s[8 * t + 5]),
                     pack_bf16x2(s[8 * t + 6], s[8 * t + 7])};
    return __builtin_bit_cast(bf16x8, w);
}

__device__ __forceinline__ float other_half(float v) {   // of lane ^ 32
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? (uint32_t)s[0] : (uint32_t)s[1]);
}

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int v = 0; v < 16; ++v) z[v] = 0.f;
    return z;
}

// Index of accumulator register v's row within its block of 32.
__device__ __forceinline__ constexpr int acc_row(int v) { return 8 * (v >> 2) + (v & 3); }

// tanh(s c) of a product s, c = scale / cap:  |tanh y| = (1 - e) / (1 + e), e = exp(-2 |y|), off by some 2^-21 of it and by what the exponential's last
// place makes, 2^-24, which the cap multiplies and which is all there is near 0.  Up to a cap of kFarCap that is 2^-18 of a score at most.  FAR: up to
// |y| = 1/8 the series y - y^3 / 3 + 2 y^5 / 15 (its next term is 2^-22 of it), so that a score is off by 2^-20 of itself whatever its cap.
constexpr float kFarCap = 64.f;
template <bool FAR>
__device__ __forceinline__ float score_tanh(float s, float c) {
    const float y = s * (c * (2.f * kLog2e)), e = __builtin_amdgcn_exp2f(-fabsf(y));
    float t = __builtin_copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), y);
    if constexpr (FAR) {
        constexpr float k = 0.5f / kLog2e, k3 = -k * k * k / 3.f, k5 = k * k * k * k * k * (2.f / 15.f), most = 0.125f / k;
        const float z = y * y, near = y * __builtin_fmaf(z, __builtin_fmaf(z, k5, k3), k);
        t = z < most * most ? near : t;
    }
    return t;
}
// Blocks of products become tanh's, in one branch that a call takes always or never (us by the branch, cap 30 / cap 1000 / the far form always; 8192 tokens, 32
// heads of 64: forward 567 / 711 / 761, backward 1623 / 1865 / 1937; 32 of 128 on 8: 773 / 892 / 881, 2507 / 2734 / 2749).  The exponentials stay outside:
// with them in the branch the backward passes of d = 128 spill, 2507 -> 2740.
template <typename... BLOCKS>
__device__ __forceinline__ void cap_scores(float cap, float c, BLOCKS&... s) {
    auto each = [&](auto far, f32x16& x) {
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = score_tanh<far.value>(x[v], c);
    };
    if (cap > kFarCap) (each(std::true_type(), s), ...);
    else (each(std::false_type(), s), ...);
}
// A score times log2(e): from the product s, c = scale log2(e); capped: from s = tanh, factor = 1 - tanh^2.
template <bool CAP>
__device__ __forceinline__ float score_log2(float s, float c, float cap_log2e, float& factor) {
    factor = CAP ? __builtin_fmaf(-s, s, 1.f) : 1.f;
    return CAP ? cap_log2e * s : s * c;
}

// Columns of a transposed result (acc[b]: elements 32 b .. 32 b + 31 of a row of d, the row being this lane's column): 16-byte pieces.
template <int NB>
__device__ __forceinline__ void store_columns(const f32x16 (&acc)[NB], float factor, uint16_t* row, int d, bool mine, int lane) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            uint32_t x[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    x[i][e] = pack_bf16x2(acc[b][4 * (j + i) + 2 * e] * factor, acc[b][4 * (j + i) + 2 * e + 1] * factor);
            // the halves of the wave hold 4 elements of each 8: after the exchange one has the first 8, the other the next
            const auto lo = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
            const int at = 32 * b + 8 * (j + (lane >> 5));
            const u32x4 w = {(uint32_t)lo[0], (uint32_t)hi[0], (uint32_t)lo[1], (uint32_t)hi[1]};
            if (mine && at < d) *reinterpret_cast<u32x4*>(row + at) = w;
        }
}

// The same as a part's sums: fp32, elements from row on.
template <int NB>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[NB], float* row, int d, bool mine, int lane) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = 32 * b + 8 * j + 4 * (lane >> 5);
            const f32x4 x = {acc[b][4 * j], acc[b][4 * j + 1], acc[b][4 * j + 2], acc[b][4 * j + 3]};
            if (mine && at < d) *reinterpret_cast<f32x4*>(row + at) = x;
        }
}

}  // namespace qg
