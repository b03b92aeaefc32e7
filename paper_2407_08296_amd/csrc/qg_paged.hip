// Attention of one new token per sequence over a cache in pages: o = softmax_j(x_j) v_j over positions j = first .. length - 1.
// The cache is read once, 4 d bytes per key head and position: HBM is the bound, and what counts is how many bytes are on their way.  The
// query heads that share a key head are taken together, up to 16 as the columns of a 16 x 16 x 32 product (one alone leaves 15
// columns empty: at 8 TB/s that is still 5 % of the matrix pipe).  A sequence is cut into parts for many workgroups,
// whose results are joined by a second kernel; a workgroup's waves take 32 positions each in turn, each with tiles, maximum and sums of
// its own, so that nothing waits for another wave before the end.
//   K straight into operands: lane l holds position l % 16 and 8 elements of d.  V by direct loads into LDS (rows as in qg_attention.h), read
// transposed.  Scores are [position][head]; register i of block b is position 16 b + 4 (l / 16) + i, the order in which V is read then.
// us and what that is of a large copy's rate (4.9 TB/s): one sequence of 32768, 8 key heads of 128, 30 + 4.4 for the join (91 % without it); 8 of up
// to 8000, 32 key heads of 128, 87 (5.0 TB/s with the join); 64 of up to 4096, 16 of 64, capped, windowed, 33.5 + 4.5 (76 % without it).
#include "qg_attention.h"

namespace qg {

constexpr int kPagedStep = 32;              // positions of a wave at a time

struct PagedArgs {
    const uint16_t *q, *k, *v;
    uint16_t* o;
    const int32_t *table, *lengths;
    const float* slopes;
    float* part;                            // [sequences][heads_q][shares][d] sums, then [..][2]: maximum (log2), sum
    int64_t q_ts, q_hs, o_ts, o_hs, pages;
    int page_size, heads_k, group, d, sequences, width, part_length, shares, window;     // shares: workgroups that take a sequence's parts in turn
    float scale, cap;
};

// Visible positions of a sequence, and their parts, which begin at whole steps: one at least, so that a sequence without any gets its zeros.
__device__ __forceinline__ void paged_range(const PagedArgs& a, int seq, int& first, int& end) {
    end = (int)min((int64_t)max(a.lengths[seq], 0), (int64_t)a.width * a.page_size);
    first = a.window > 0 ? max(0, end - a.window) : 0;
}
__device__ __forceinline__ int paged_parts(const PagedArgs& a, int first, int end) {
    return max(1, (end - first / kPagedStep * kPagedStep + a.part_length - 1) / a.part_length);
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_paged(PagedArgs a) {
    constexpr int P = D <= 64 ? 64 : 128, NB = D / 16, NS = D / 32, CPR = P / 8, LOADS = kPagedStep * CPR / 64, PER = 64 / CPR;
    constexpr int TILE = kPagedStep * P;
    // V tiles, two per wave; at the end the waves' results, 16 rows of D (and a pad) and their maxima and sums
    constexpr int ROW = D + 4;
    static_assert(4 * 16 * ROW * 4 + 4 * 32 * 4 <= 4 * 2 * TILE * 2, "the results fit where the tiles were");
    __shared__ __attribute__((aligned(16))) uint16_t smem[4 * 2 * TILE];
    // the first shares of all sequences and heads, then the second ...: workgroups go to the 8 XCDs in turn, and with a sequence's shares next to each
    // other the first ones, which have work, would be the same XCD's (64 of up to 4096, eight shares: 65 us against 30)
    const int groups = (a.group + 15) / 16, units = a.sequences * a.heads_k * groups;
    const int part0 = blockIdx.x / units, at = blockIdx.x - part0 * units;
    // ... and of every eight units another to each XCD from one part and eight to the next: with heads of 64 an XCD that always had the same one read
    // every eighth 128-byte line, from few channels of its L2 (one of 130000, 8 heads: 64 us against 57).  The eights take turns from part to part too: an
    // XCD's workgroups go to its four engines in turn, and a long sequence among four (sixteen) short ones would have one engine of each
    // (4 of up to 30000, 8 key heads of 128: 64 us against 35; 16 of up to 16000: 75 / 59; 64 of up to 4096, 16 of 64: 38.6 / 36.3).  Two eights would come
    // around in step with the four parts (2 of up to 16000, 8 key heads of 128: 23.9 / 22.7; taking turns every second part with 24 and 32 units too: of
    // 16 calls two changed by more than a hundredth, 4 of up to 30000, 8 key heads, 36.2 / 35.1, 4 of 7500 27.8 / 27.4).
    int unit = at;
    if ((at | 7) < units) {
        const int eight = ((at >> 3) + (units == 16 ? part0 >> 1 : part0)) % (units >> 3);
        unit = 8 * eight + ((at + eight + part0) & 7);
    }
    const int hg = unit % groups, kv = unit / groups % a.heads_k, seq = unit / groups / a.heads_k;
    int first, end;
    paged_range(a, seq, first, end);
    const int parts = paged_parts(a, first, end);
    if (part0 >= parts) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int head = kv * a.group + hg * 16 + col;
    const bool has_head = hg * 16 + col < a.group;
    const int64_t row = (int64_t)a.heads_k * a.d;
    const uint16_t *kp = a.k + (int64_t)kv * a.d, *vp = a.v + (int64_t)kv * a.d;
    const int32_t* pages = a.table + (int64_t)seq * a.width;

    bf16x8 qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int c = 4 * s + g;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (has_head && c * 8 < a.d) w = *reinterpret_cast<const u32x4*>(a.q + (int64_t)seq * a.q_ts + (int64_t)head * a.q_hs + c * 8);
        qf[s] = __builtin_bit_cast(bf16x8, w);
    }
    const float c2 = CAP ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
    const float slope = BIAS && has_head ? a.slopes[head] * kLog2e : 0.f;

    // row of the cache that the wave's step holds at position lane % 32, -1: none (hidden, past the end, or without a page)
    auto slot_of = [&](int j0) {
        const int j = j0 + (lane & 31);
        if (j < first || j >= end) return -1;
        const int at = (int)((uint32_t)j / (uint32_t)a.page_size), page = pages[at];
        return page < 0 || page >= a.pages ? -1 : page * a.page_size + (j - at * a.page_size);
    };
    uint16_t* const tiles = smem + wave * 2 * TILE;
    bf16x8 kf[2][2][NS];
    auto fetch = [&](int slot, int stage, bf16x8 (&to)[2][NS]) {
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int r = p * PER + lane / CPR, chunk = (lane % CPR) ^ tile_swizzle<P>(r);
            const int from = max(0, __shfl(slot, r, 64));
            const uint16_t* src = vp + (int64_t)from * row + (chunk * 8 < a.d ? chunk * 8 : 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             (__attribute__((address_space(3))) void*)(tiles + stage * TILE + p * 512), 16, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int from = max(0, __shfl(slot, 16 * b + col, 64));
            const uint16_t* src = kp + (int64_t)from * row;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int c = 4 * s + g;
                u32x4 w = *reinterpret_cast<const u32x4*>(src + (c * 8 < a.d ? c * 8 : 0));
                to[b][s] = __builtin_bit_cast(bf16x8, w);
            }
        }
    };
    f32x4 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    auto compute = [&](int j0, uint32_t there, int stage, const bf16x8 (&kk)[2][NS]) {
        uint16_t* V = tiles + stage * TILE;
        if (there != 0xFFFFFFFFu) {          // rows without a position: zero, whatever was read
#pragma unroll
            for (int p = 0; p < LOADS; ++p) {
                const int r = p * PER + lane / CPR;
                if (!(there >> r & 1)) *reinterpret_cast<u32x4*>(V + p * 512 + lane * 8) = u32x4{0u, 0u, 0u, 0u};
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        f32x4 s[2];
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NS; ++k) s[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[b][k], qf[k], s[b], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (the far form whatever the cap: 64 of up to 4096, 16 of 64, 36.0 -> 36.8 us; a branch for the near one needs more than 128 registers, 39.1)
                float unused, x = score_log2<CAP>(CAP ? score_tanh<true>(s[b][i], c2) : s[b][i], c2, cap2, unused);
                const int r = 16 * b + 4 * g + i;
                if constexpr (BIAS) x = __builtin_fmaf(-slope, (float)(end - 1 - (j0 + r)), x);
                s[b][i] = there >> r & 1 ? x : -INFINITY;
                top = fmaxf(top, s[b][i]);
            }
        }
        if (__ballot(top > m + 8.f) != 0) {
            top = fmaxf(top, __shfl_xor(top, 16, 64));
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float raised = fmaxf(m, top);
            const float keep = raised == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - raised);
            m = raised;
            l *= keep;
#pragma unroll
            for (int b = 0; b < NB; ++b) o[b] *= keep;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[b][i] = __builtin_amdgcn_exp2f(s[b][i] - ref);
                l += s[b][i];
            }
        const u32x4 pw = {pack_bf16x2(s[0][0], s[0][1]), pack_bf16x2(s[0][2], s[0][3]), pack_bf16x2(s[1][0], s[1][1]), pack_bf16x2(s[1][2], s[1][3])};
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw);
        const int r = 4 * g + (col >> 2);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int chunk = 2 * b + ((col & 3) >> 1);
            const uint16_t* lo = V + r * P + ((chunk ^ tile_swizzle<P>(r)) * 8) + 4 * (col & 1);
            const uint16_t* hi = V + (r + 16) * P + ((chunk ^ tile_swizzle<P>(r + 16)) * 8) + 4 * (col & 1);
            const s16x4 x = lds_read_tr((lds_s16x4*)lo);
            const s16x4 y = lds_read_tr((lds_s16x4*)hi);
            const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
            o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf, o[b], 0, 0, 0);
        }
    };
    // the wave's own LDS accesses and direct loads complete in order once waited for; the scheduler does not see the transposing reads as accesses
    auto fence = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    // The wave's steps: of each part of this share every fourth; the last part of a sequence may end early.
    const int by = 4 * kPagedStep, per = a.part_length / by, base = first / kPagedStep * kPagedStep + wave * kPagedStep;
    const int mine = (parts - part0 + a.shares - 1) / a.shares, last = part0 + (mine - 1) * a.shares;
    const int steps = (mine - 1) * per + min(max((end - base - last * a.part_length + by - 1) / by, 0), per);
    auto position = [&](int i) {
        const int part = i / per;
        return base + (part0 + part * a.shares) * a.part_length + (i - part * per) * by;
    };
    int slot = steps > 0 ? slot_of(position(0)) : -1, next = steps > 1 ? slot_of(position(1)) : -1;
    if (steps > 0) fetch(slot, 0, kf[0]);
    for (int i = 0; i < steps; i += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (i + u < steps) {
                const uint32_t there = (uint32_t)__ballot(slot >= 0);
                fence();
                if (i + u + 1 < steps) {
                    fetch(next, 1 - u, kf[1 - u]);
                    slot = next;
                    next = i + u + 2 < steps ? slot_of(position(i + u + 2)) : -1;
                }
                compute(position(i + u), there, u, kf[u]);
            }
        }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    // join the waves: columns of heads, in a fixed order
    lds_barrier();
    float* sums = reinterpret_cast<float*>(smem);                // [wave][16][ROW]
    float* stat = sums + 4 * 16 * ROW;                           // [wave][16][2]
#pragma unroll
    for (int b = 0; b < NB; ++b) *reinterpret_cast<f32x4*>(sums + (wave * 16 + col) * ROW + 16 * b + 4 * g) = o[b];
    if (g == 0) {
        stat[(wave * 16 + col) * 2] = m;
        stat[(wave * 16 + col) * 2 + 1] = l;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * (D / 4); idx += 256) {
        const int q = idx / (D / 4), e = idx % (D / 4) * 4;
        if (hg * 16 + q >= a.group || e >= a.d) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[(w * 16 + q) * 2]);
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(stat[(w * 16 + q) * 2] - ref);
            sum = __builtin_fmaf(stat[(w * 16 + q) * 2 + 1], f, sum);
            x += *reinterpret_cast<const f32x4*>(sums + (w * 16 + q) * ROW + e) * f;
        }
        const int h = kv * a.group + hg * 16 + q;
        if (a.shares == 1) {
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            uint32_t* to = reinterpret_cast<uint32_t*>(a.o + (int64_t)seq * a.o_ts + (int64_t)h * a.o_hs + e);
            to[0] = pack_bf16x2(x[0] * f, x[1] * f);
            to[1] = pack_bf16x2(x[2] * f, x[3] * f);
        } else {
            const int64_t row = ((int64_t)seq * a.heads_k * a.group + h) * a.shares + part0;
            *reinterpret_cast<f32x4*>(a.part + row * a.d + e) = x;
            if (e == 0) {
                float* to = a.part + (int64_t)a.sequences * a.heads_k * a.group * a.shares * a.d + 2 * row;
                to[0] = top;
                to[1] = sum;
            }
        }
    }
}

// Joins the shares of a sequence's heads in a fixed order: WAVES waves per head, of each 64 / (d / 4) shares at once, four elements per lane.
template <int WAVES>
__global__ __launch_bounds__(WAVES > 4 ? 64 * WAVES : 256) void k_attention_join(PagedArgs a) {
    constexpr int HEADS = WAVES > 4 ? 1 : 4 / WAVES;
    __shared__ __attribute__((aligned(16))) float sums[HEADS * WAVES][128 + 4];
    const int heads = a.heads_k * a.group, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % WAVES;
    const int64_t unit = min((int64_t)blockIdx.x * HEADS + wave / WAVES, (int64_t)a.sequences * heads - 1);
    const int seq = (int)(unit / heads), h = (int)(unit - (int64_t)seq * heads);
    int first, end;
    paged_range(a, seq, first, end);
    const int parts = min(a.shares, paged_parts(a, first, end));
    const float *from = a.part + unit * a.shares * a.d, *stat = a.part + (int64_t)a.sequences * heads * a.shares * a.d + 2 * unit * a.shares;
    const int per = a.d / 4, at_once = 64 / per, e = lane % per * 4, mine = lane / per;
    float top = -INFINITY;
    for (int p = lane; p < parts; p += 64) top = fmaxf(top, stat[2 * p]);
    top = wave_max(top);
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    if (mine < at_once)
#pragma unroll 4
        for (int p = w * at_once + mine; p < parts; p += WAVES * at_once) {
            const float f = __builtin_amdgcn_exp2f(stat[2 * p] - ref);
            sum = __builtin_fmaf(stat[2 * p + 1], f, sum);
            x += *reinterpret_cast<const f32x4*>(from + (int64_t)p * a.d + e) * f;
        }
    // the shares of a wave, then the waves
    float y[5] = {x[0], x[1], x[2], x[3], sum};
    for (int o = 1; o < at_once; ++o)
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const float v = __shfl(i < 4 ? x[i & 3] : sum, lane % per + o * per, 64);
            y[i] += v;
        }
    if constexpr (WAVES > 1) {
        if (mine == 0) *reinterpret_cast<f32x4*>(&sums[wave][e]) = f32x4{y[0], y[1], y[2], y[3]};
        if (lane == 0) sums[wave][128] = y[4];
        __syncthreads();
        if (w != 0) return;
#pragma unroll
        for (int o = 1; o < WAVES; ++o) {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += sums[wave + o][min(e, 124) + i];
            y[4] += sums[wave + o][128];
        }
    }
    if (mine != 0) return;
    const float f = y[4] == 0.f ? 0.f : 1.f / y[4];
    const u32x2 o = {pack_bf16x2(y[0] * f, y[1] * f), pack_bf16x2(y[2] * f, y[3] * f)};
    *reinterpret_cast<u32x2*>(a.o + (int64_t)seq * a.o_ts + (int64_t)h * a.o_hs + e) = o;
}

// Positions of a workgroup: 512, and 256 where that leaves fewer than 512 workgroups (us with 256 / 512 / 1024: 128 sequences of up to 1000, 8 heads
// on one: 14.7 / 16.4 / 16.4; 64 of up to 4096, 16 of 64: - / 37.1 / 39.5; 8 of up to 8000, 32 of 128: - / 136 / 138).  One sequence's parts are all
// of one length: as many as fill the chip's 512 places in as few whole rounds as parts of at most 512 make (us with the rule for several / this
// one: 20000 positions, 8 key heads of 128: 24.0 / 22.3; 36000: 41.6 / 36.8; 100000, two: 33.4 / 29.4; 200000, one: 38.6 / 30.9; parts of up to 1024: 50000,
// eight, 53.4 -> 49.0, but 100000, 8 of 64, 49.9 -> 55.9.  10 sequences of up to 10000, two: 15.7 / 19.1; two to four sequences by this rule, the rule
// for several / this one: 2 of 50000, two, 28.1 / 25.0; 4 of 9000, eight, 33.5 / 31.7; 3 of 4000, 16 of 64, 16.0 / 16.4; one of 20000 and three of a tenth, eight,
// 25.6 / 25.5).  A window may begin inside a step, so a table is taken to hold one part more than its length has; without a window that one has no work (32768
// positions, 8 key heads, fill 512 places and launch 520: 29.3 us, 512 of them and the join for up to 64 shares 29.1).
static int part_length(const qg_cache* c, int heads_q) {
    const int64_t units = (int64_t)c->sequences * c->heads * ((heads_q / c->heads + 15) / 16), all = units * c->width * c->page_size;
    if (c->sequences > 1) return all < 512 * 512 ? 256 : 512;
    const int64_t rounds = (all + 512 * 512 - 1) / (512 * 512), fit = (all + 512 * rounds - 1) / (512 * rounds);
    return fit <= 256 ? 256 : (int)((fit + 4 * kPagedStep - 1) / (4 * kPagedStep) * (4 * kPagedStep));
}
static int64_t most_parts(const qg_cache* c, int heads_q) {
    const int length = part_length(c, heads_q);
    return ((int64_t)c->width * c->page_size + kPagedStep - 1 + length - 1) / length;
}
// Workgroups per sequence and key head: all parts, but no more than make 8192 in all (a table is as wide as the longest sequence may get: 64 sequences of
// 1000 positions, 8 key heads, in a table for 131072, one workgroup for each part 143 us, of which most had nothing to do; 200 of up to 1000, 32 key heads, one workgroup for both parts 54.5, two and their
// join 63.6; with 4096 in all 128 of up to 4096, 16 key heads, 53.6 -> 63.4).  So beyond 4096 sequences and key heads one workgroup walks all parts, long ones
// too: 512 / 513 sequences of 300, 8 key heads of 128, and one of 32768 among them, 370 / 503; with 65536 workgroups in all 248 / 269, but 513 and one of 4000
// 127 -> 182, 1000 of 500 354 -> 400, 700 of up to 1000 257 -> 301.
static int64_t most_shares(const qg_cache* c, int heads_q) {
    const int64_t units = (int64_t)c->sequences * c->heads * ((heads_q / c->heads + 15) / 16), parts = most_parts(c, heads_q);
    const int64_t shares = units < 8192 ? 8192 / units : 1;
    return shares < parts ? shares : parts;
}

static int check_paged(const qg_cache* c, int heads_q) {
    if (int e = check_cache(c)) return e;
    if (c->d > 128 || heads_q <= 0 || heads_q > kAttnMaxHeads || heads_q % c->heads != 0) return QG_ERR_SHAPE;
    if ((int64_t)c->sequences * heads_q >= (int64_t(1) << 24)) return QG_ERR_SHAPE;   // (2^32 threads in a launch)
    return QG_OK;
}

}  // namespace qg

using namespace qg;

extern "C" size_t qg_attention_paged_workspace_bytes(const qg_cache* c, int heads_q) {
    if (check_paged(c, heads_q) != QG_OK) return 0;
    return ((size_t)most_shares(c, heads_q) * c->sequences * heads_q * (c->d + 2) * 4 + 15) / 16 * 16;
}

extern "C" int qg_attention_paged(const qg_cache* c, const int32_t* lengths, const qg_heads* q, int heads_q, float scale, float cap, int64_t window,
                                  const float* slopes, const qg_heads* o, void* workspace, size_t workspace_bytes, void* stream) {
    if (int e = check_paged(c, heads_q)) return e;
    if (lengths == nullptr) return QG_ERR_NULL;
    for (const qg_heads* x : {q, o})
        if (int e = check_heads(x, true)) return e;
    if (!check_scores(scale, cap) || window < 0) return QG_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(lengths) & 3) || (reinterpret_cast<uintptr_t>(slopes) & 3) || !aligned16(workspace)) return QG_ERR_ALIGN;
    if (workspace == nullptr || workspace_bytes < qg_attention_paged_workspace_bytes(c, heads_q)) return QG_ERR_WORKSPACE;
    PagedArgs a = {};
    a.q = q->data, a.q_ts = q->token_stride, a.q_hs = q->head_stride;
    a.o = o->data, a.o_ts = o->token_stride, a.o_hs = o->head_stride;
    a.k = c->k, a.v = c->v, a.table = c->table, a.lengths = lengths, a.slopes = slopes, a.part = static_cast<float*>(workspace);
    a.pages = c->pages, a.page_size = c->page_size, a.heads_k = c->heads, a.group = heads_q / c->heads, a.d = c->d;
    a.sequences = c->sequences, a.width = c->width, a.part_length = part_length(c, heads_q);
    a.shares = (int)most_shares(c, heads_q);
    a.window = (int)(window < (int64_t(1) << 31) ? window : 0);
    a.scale = scale, a.cap = cap;
    const unsigned grid = (unsigned)((int64_t)a.shares * a.sequences * a.heads_k * ((a.group + 15) / 16));
    auto launch = [&](auto d, auto cp, auto bias) {
        hipLaunchKernelGGL((k_attention_paged<d.value, cp.value, bias.value>), dim3(grid), dim3(256), 0, (hipStream_t)stream, a);
    };
    auto with_d = [&](auto cp, auto bias) {
        if (a.d <= 64) launch(std::integral_constant<int, 64>(), cp, bias);
        else if (a.d <= 96) launch(std::integral_constant<int, 96>(), cp, bias);     // (as 128: 50000 positions, 8 key heads of 96, 43.2 -> 44.8 us, 16 of up to 2000, 72, 16.6 -> 18.4)
        else launch(std::integral_constant<int, 128>(), cp, bias);
    };
    auto with_bias = [&](auto cp) { slopes != nullptr ? with_d(cp, std::true_type()) : with_d(cp, std::false_type()); };
    cap > 0.f ? with_bias(std::true_type()) : with_bias(std::false_type());
    const int64_t heads = (int64_t)a.sequences * heads_q;
    // (one wave, four, sixteen per head; 100000 positions, 16 heads on two, 390 shares: four 35.7, sixteen 33.4)
    if (a.shares > 64) hipLaunchKernelGGL(k_attention_join<16>, dim3((unsigned)heads), dim3(1024), 0, (hipStream_t)stream, a);
    else if (a.shares > 16) hipLaunchKernelGGL(k_attention_join<4>, dim3((unsigned)heads), dim3(256), 0, (hipStream_t)stream, a);
    else if (a.shares > 1) hipLaunchKernelGGL(k_attention_join<1>, dim3((unsigned)((heads + 3) / 4)), dim3(256), 0, (hipStream_t)stream, a);
    return check_launch();
}
