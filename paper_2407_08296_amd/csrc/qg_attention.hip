// Attention over packed sequences, forward and backward.  With x = scale q.k, capped cap tanh(x / cap), minus slope |distance|, over the
// visible keys of a query (qg_attention.h):
//     lse = log sum_j exp(x_j),   p_j = exp(x_j - lse),   o = sum_j p_j v_j
//     delta = sum_d do o,   ds_j = p_j (do.v_j - delta) (1 - tanh^2) scale
//     dq = sum_j ds_j k_j,   dk_j = sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i
// One pass over the keys with a running maximum and sum; exponentials to the base 2.  p and ds are rounded to bf16, operands of
// matrix products, as every product of the library has them; maxima, sums, lse, delta and all accumulators are fp32.
// Backward: one kernel for dq (queries stay, keys pass by) and one for dk and dv (keys stay, queries of all heads that share them
// pass by): eight products where one kernel would do five, but each sum has one owner and one order: no atomics, the same bits every time.
// o is stored in bf16, and a delta from that is off by a rounding of sum do o in all of a row (dq and dk off by 0.0031 of their size at 64 keys, 0.0028 at
// 512, where their own roundings make 0.0024).  But the true p_j (do.v_j - delta) add up to 0 over a row: what they come to, r, is what delta
// lacks.  So the pass for dq also forms r and the mean key k' = sum_j p_j (1 - tanh^2) k_j, takes r k' off in the end and leaves delta + r for dk:
// a product more, from operands that are there (8192 tokens, 32 heads of 128 on 8: dq 924 -> 1020 us).
//
// What bounds them: the matrix pipe at the clock it holds under such a load, and the operands' way to it.  Forward, 8192 tokens, 16 heads of 128, no mask: 552 us;
// the products alone, on operands in registers, 405 (1355 TFLOP/s); with the softmax 437; with LDS reads and no softmax 466; all but the direct loads 510.
// By counters (4096 tokens, 16 heads, no mask; matrix pipe + vector instructions, of the time): d = 128 forward 53 + 51 %, dq 67 + 50 %, dkv 54 + 33 %; d = 64
// 36 + 59 %, 50 + 56 %, 46 + 41 %; LDS is busy for 18 to 40 %, without bank conflicts; with a cap 32 + 70 %, 45 + 69 %, 40 + 55 % and 20 + 82 %, 28 + 77 %,
// 28 + 68 %.  Gains nothing (us, 8192 tokens, 32 heads of 128 on 8, forward):
// a step's exponentials interleaved with the next step's products by hand 546 -> 558; 64 queries per wave 559 -> 703; 8 waves and 256 queries per
// workgroup 564 -> 565, and 35 -> 45 for sequences of 315 tokens.
// us (PFLOP/s by 4 and 10 d per visible pair; 8192 tokens, causal): 32 heads of 128 on 8, one sequence: forward 549 (1.0), backward 1992 (0.69); 32 on 32, two
// sequences: 322 (0.91), 1165 (0.63); 32 heads of 64, one sequence: 350 (0.78), 1091 (0.63); 5 % more on another card.  The vendor's product of 8192^3: 1.2.
#include "qg_attention.h"

namespace qg {

constexpr int kAttnWaves = 4;      // of a workgroup, 32 rows each
constexpr int kAttnRows = 32 * kAttnWaves;
constexpr int kAttnStep = 64;      // rows that pass by, per step

template <int D>
constexpr int attn_pitch() { return D <= 64 ? 64 : 128; }
// Rows per step of the backward passes: beyond d = 64, 32 of them leave room in LDS for dO's (V's) rows and a second workgroup.  (Three or four steps in
// LDS instead of two: the same times for 16 sequences of 256 tokens and for one of 8192.)
template <int D>
constexpr int attn_back_step() { return D <= 64 ? 64 : 32; }

// What the scores of a query (or of a key's queries) need.
struct ScoreRule {
    float c, cap_log2e, slope;
};
template <bool CAP, bool BIAS>
__device__ __forceinline__ ScoreRule score_rule(const AttnArgs& a, int head) {
    ScoreRule r;
    r.c = CAP ? a.scale / a.cap : a.scale * kLog2e;
    r.cap_log2e = a.cap * kLog2e;
    r.slope = BIAS ? a.slopes[head] * kLog2e : 0.f;
    return r;
}

// Visible keys lo .. hi of the query at row i of a sequence.
struct Visible {
    int shift, last, causal, prefix, window;
    __device__ __forceinline__ Visible(const AttnArgs& a, const AttnTile& t) {
        shift = t.nk - t.nq;
        last = t.nk - 1;
        causal = a.causal;
        prefix = t.prefix;
        window = a.window;
    }
    __device__ __forceinline__ int hi(int i) const { return causal ? min(last, max(i + shift, prefix - 1)) : last; }
    __device__ __forceinline__ int lo(int i) const { return window > 0 ? max(0, i + shift - window + 1) : 0; }
};

// Forward: 128 queries per workgroup, 32 per wave, in registers; keys and values pass by in steps of 64 through two stages of LDS.  A wave's scores are
// transposed ([key][query]), so that a query's maximum and sum are its lane's, and probabilities become operands as they lie.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_fwd(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16;
    __shared__ __attribute__((aligned(256))) uint16_t smem[4 * kAttnStep * P];
    int head, t, part;
    if (!attn_place(a.heads_q, a.tiles, a.parts, head, t, part)) return;
    const AttnTile seq = attn_tile<kAttnRows, false>(a, a.tiles - 1 - t);   // late tiles first: with a causal mask they have most keys
    const int row0 = seq.tile * kAttnRows;
    if (row0 < 0 || row0 >= seq.nq) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const ScoreRule rule = score_rule<CAP, BIAS>(a, head);
    const int kv = head / a.group;
    const uint16_t* qp = a.q + (int64_t)(seq.q0 + row0) * a.q_ts + (int64_t)head * a.q_hs;
    const uint16_t* kp = a.k + (int64_t)seq.k0 * a.k_ts + (int64_t)kv * a.k_hs;
    const uint16_t* vp = a.v + (int64_t)seq.k0 * a.v_ts + (int64_t)kv * a.v_hs;

    const int w0 = row0 + 32 * wave, i = w0 + (lane & 31), w1 = min(w0 + 31, seq.nq - 1);
    bf16x8 qf[NS];
    const RowFrags qr(qp, a.q_ts, wave, lane, i < seq.nq, a.d);
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = qr.get(s);
    const int lo = see.lo(i), hi = see.hi(i);
    // steps that some row of the workgroup sees, of them the part's; and, of the wave, those that all rows see whole
    const int first = see.lo(row0) / kAttnStep, most = see.hi(min(row0 + kAttnRows, seq.nq) - 1);
    const int all = most < 0 ? 0 : most / kAttnStep - first + 1;
    int begin, steps;
    attn_share(all, a.parts, part, begin, steps);
    const int wave_lo = see.lo(w0), wave_hi = w0 < seq.nq ? see.hi(w1) : -1, all_lo = see.lo(w1), all_hi = see.hi(w0);

    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = zero16();
    float m = -INFINITY, l = 0.f;       // running maximum (as it was when last raised) and the lane's part of the sum

    RowsTile<P, kAttnStep, 256> kt, vt;
    kt.init(a.k_ts, a.d);
    vt.init(a.v_ts, a.d);
    auto fetch = [&](int step, int stage) {
        const int j = (first + step) * kAttnStep;
        kt.load(smem + stage * 2 * kAttnStep * P, kp + (int64_t)j * a.k_ts, a.k_ts, seq.nk - j);
        vt.load(smem + (stage * 2 + 1) * kAttnStep * P, vp + (int64_t)j * a.v_ts, a.v_ts, seq.nk - j);
    };
    const float pos = (float)(i + see.shift - 4 * h);     // from the register's key without its 4 h
    using Reader = TileReader<P>;
    const Reader reader(lane);
    auto compute = [&](int j0, uint32_t tile, bool masked) {       // tile: K's rows, V's behind them
        const uint32_t kr = tile + reader.rows, vc = tile + kAttnStep * P * 2 + reader.columns;
        f32x16 s[2];
        __builtin_amdgcn_s_setprio(kMfmaPrio);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = zero16();
#pragma unroll
            for (int k = 0; k < NS; ++k) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Reader::frag(kr, 32 * b, k), qf[k], s[b], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        constexpr bool kScaled = CAP || BIAS;     // s holds x log2(e) then
        float top = -INFINITY;
        if constexpr (kScaled) {
            const float away = pos - (float)j0;
            if constexpr (CAP) cap_scores(a.cap, rule.c, s[0], s[1]);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    float unused;
                    s[b][v] = score_log2<CAP>(s[b][v], rule.c, rule.cap_log2e, unused);
                    if constexpr (BIAS) s[b][v] = __builtin_fmaf(-rule.slope, fabsf(away - (float)(32 * b + acc_row(v))), s[b][v]);
                }
        }
        if (masked) {     // (a branch around the selects alone: with a masked and a plain body the registers of both spill)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int j = j0 + 32 * b + acc_row(v) + 4 * h;
                    s[b][v] = j >= lo && j <= hi ? s[b][v] : -INFINITY;
                }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) top = fmaxf(top, s[b][v]);
        top = fmaxf(top, other_half(top));
        if constexpr (!kScaled) top *= rule.c;
        // any reference near the maximum serves: it is raised only when the terms would pass 2^8 (the accumulators are rescaled then)
        if (__ballot(top > m + 8.f) != 0) {
            const float raised = fmaxf(m, top);
            const float keep = raised == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - raised);
            m = raised;
            l *= keep;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[b][v] *= keep;
        }
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float x = kScaled ? s[b][v] - ref : __builtin_fmaf(s[b][v], rule.c, -ref);
                s[b][v] = __builtin_amdgcn_exp2f(x);
                l += s[b][v];
            }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 pf = score_frag(s[b], u);
#pragma unroll
                for (int c = 0; c < NB; ++c)
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Reader::frag_t(vc, 32 * b + 16 * u, c), pf, o[c], 0, 0, 0);
            }
    };

    if (steps > begin) fetch(begin, begin & 1);
    for (int step = begin; step < steps; ++step) {
        wait_loads<0>();
        lds_barrier();
        if (step + 1 < steps) fetch(step + 1, (step + 1) & 1);
        const int j0 = (first + step) * kAttnStep;
        if (j0 > wave_hi || j0 + kAttnStep <= wave_lo) continue;
        compute(j0, tile_address(smem) + (step & 1) * 4 * kAttnStep * P, j0 < all_lo || j0 + kAttnStep - 1 > all_hi);
    }
    l += other_half(l);
    const bool mine = i < seq.nq;
    if (a.parts > 1) {
        const int64_t row = ((int64_t)part * a.heads_q + head) * a.tokens_q + seq.q0 + i, rows = (int64_t)a.parts * a.heads_q * a.tokens_q;
        store_part(o, a.part + row * a.d, a.d, mine, lane);
        if (mine && h == 0) {
            a.part[rows * a.d + 2 * row] = m;
            a.part[rows * a.d + 2 * row + 1] = l;
        }
        return;
    }
    if (mine && h == 0 && a.lse != nullptr)
        a.lse[(int64_t)head * a.tokens_q + seq.q0 + i] = l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    store_columns(o, l == 0.f ? 0.f : 1.f / l, a.o + (int64_t)(seq.q0 + i) * a.o_ts + (int64_t)head * a.o_hs, a.d, mine, lane);
}

// Joins the parts of the forward pass in their order: four elements of a row per thread.
__global__ __launch_bounds__(256) void k_attention_fwd_join(AttnArgs a) {
    const int per = a.d / 4;
    const int64_t rows = (int64_t)a.heads_q * a.tokens_q, at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / per;
    if (row >= rows) return;
    const int e = (int)(at - row * per) * 4, head = (int)(row / a.tokens_q), token = (int)(row - (int64_t)head * a.tokens_q);
    const float* stat = a.part + rows * a.parts * a.d + 2 * row;
    float top = -INFINITY, sum = 0.f;
    for (int p = 0; p < a.parts; ++p) top = fmaxf(top, stat[2 * rows * p]);
    const float ref = top == -INFINITY ? 0.f : top;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < a.parts; ++p) {
        const float f = __builtin_amdgcn_exp2f(stat[2 * rows * p] - ref);
        sum = __builtin_fmaf(stat[2 * rows * p + 1], f, sum);
        x += *reinterpret_cast<const f32x4*>(a.part + (rows * p + row) * a.d + e) * f;
    }
    if (e == 0 && a.lse != nullptr) a.lse[row] = sum > 0.f || sum != sum ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    const u32x2 w = {pack_bf16x2(x[0] * f, x[1] * f), pack_bf16x2(x[2] * f, x[3] * f)};
    *reinterpret_cast<u32x2*>(a.o + (int64_t)token * a.o_ts + (int64_t)head * a.o_hs + e) = w;
}

// s, a product (capped: its tanh), becomes p = exp2(x - lse), the exponent being s c + offset where x is linear in it and x + offset else; dp, less delta, becomes p (dp -
// delta).  Returns what that is multiplied by for the gradient of scale q.k (1 - tanh^2, or 1).
template <bool CAP, bool BIAS>
__device__ __forceinline__ float score_gradient(float& s, float& dp, const ScoreRule& rule, float offset, float distance) {
    float factor = 1.f;
    if constexpr (!CAP && !BIAS) {
        s = __builtin_amdgcn_exp2f(__builtin_fmaf(s, rule.c, offset));
    } else {
        float x = score_log2<CAP>(s, rule.c, rule.cap_log2e, factor);
        if constexpr (BIAS) x = __builtin_fmaf(-rule.slope, fabsf(distance), x);
        s = __builtin_amdgcn_exp2f(x + offset);
    }
    dp *= s;
    return factor;
}

// dq, in the forward pass's shape.  From d = 65 on dO's rows are parked in LDS (registers: dq and the mean key 64 each, q 32, a block of scores and their
// gradients 32), and one block of 32 x 32 scores is worked on at a time, its operands read one ahead.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_dq(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16, STEP = attn_back_step<D>();
    constexpr bool PARKED = D > 64;
    __shared__ __attribute__((aligned(256))) uint16_t smem[4 * STEP * P + (PARKED ? kAttnRows * P : 0)];
    uint16_t* const parked = smem + 4 * STEP * P;
    int head, t, part;
    if (!attn_place(a.heads_q, a.tiles, a.parts, head, t, part)) return;
    const AttnTile seq = attn_tile<kAttnRows, false>(a, a.tiles - 1 - t);
    const int row0 = seq.tile * kAttnRows;
    if (row0 < 0 || row0 >= seq.nq) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const ScoreRule rule = score_rule<CAP, BIAS>(a, head);
    const int kv = head / a.group;
    const uint16_t* kp = a.k + (int64_t)seq.k0 * a.k_ts + (int64_t)kv * a.k_hs;
    const uint16_t* vp = a.v + (int64_t)seq.k0 * a.v_ts + (int64_t)kv * a.v_hs;
    const int w0 = row0 + 32 * wave, i = w0 + (lane & 31), w1 = min(w0 + 31, seq.nq - 1);
    const bool mine = i < seq.nq;
    const int lo = see.lo(i), hi = see.hi(i);
    const int first = see.lo(row0) / STEP, most = see.hi(min(row0 + kAttnRows, seq.nq) - 1);
    const int all = most < 0 ? 0 : most / STEP - first + 1;
    int begin, steps;
    attn_share(all, a.parts, part, begin, steps);
    const int wave_lo = see.lo(w0), wave_hi = w0 < seq.nq ? see.hi(w1) : -1, all_lo = see.lo(w1), all_hi = see.hi(w0);
    RowsTile<P, STEP, 256> kt, vt;
    kt.init(a.k_ts, a.d);
    vt.init(a.v_ts, a.d);
    auto fetch = [&](int step, int stage) {
        const int j = (first + step) * STEP;
        kt.load(smem + stage * 2 * STEP * P, kp + (int64_t)j * a.k_ts, a.k_ts, seq.nk - j);
        vt.load(smem + (stage * 2 + 1) * STEP * P, vp + (int64_t)j * a.v_ts, a.v_ts, seq.nk - j);
    };
    if (steps > begin) fetch(begin, begin & 1);      // (ahead of the rows' own loads, which delta waits for)
    const int64_t at = (int64_t)head * a.tokens_q + seq.q0 + i;
    // a row without a visible key, or none, has p = 0: its offset is -inf
    const float lse = mine ? a.lse[at] : -INFINITY, offset = lse == -INFINITY ? -INFINITY : -lse * kLog2e;
    bf16x8 qf[NS], gf[PARKED ? 1 : NS];
    float delta = 0.f;
    {
        const uint16_t* gp = a.dO + (int64_t)(seq.q0 + row0) * a.do_ts + (int64_t)head * a.do_hs;
        if constexpr (PARKED) {
            RowsTile<P, kAttnRows, 256> g;
            g.init(a.do_ts, a.d);
            g.load(parked, gp, a.do_ts, seq.nq - row0);
        }
        const RowFrags qr(a.q + (int64_t)(seq.q0 + row0) * a.q_ts + (int64_t)head * a.q_hs, a.q_ts, wave, lane, mine, a.d);
        const RowFrags gr(gp, a.do_ts, wave, lane, mine, a.d);
        const RowFrags fr(a.o + (int64_t)(seq.q0 + row0) * a.o_ts + (int64_t)head * a.o_hs, a.o_ts, wave, lane, mine, a.d);
        bf16x8 g[NS], f[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            qf[s] = qr.get(s);
            g[s] = gr.get(s);
            f[s] = fr.get(s);
        }
        __builtin_amdgcn_sched_barrier(0);     // (all on their way before the first is waited for)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if constexpr (!PARKED) gf[s] = g[s];
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)g[s][e], (float)f[s][e], delta);
        }
        delta += other_half(delta);
    }
    // For dkv, which begins its products at them, in accumulators read from LDS: -delta, and the offset in terms of the product where x is linear in it
    // (its rounding then is the one it has in the exponent too).
    auto keep_stats = [&](float d) {
        if (mine && h == 0) {
            a.stats[at] = CAP || BIAS ? offset : lse == -INFINITY ? -INFINITY : -lse / a.scale;
            a.stats[(int64_t)a.heads_q * a.tokens_q + at] = -d;
        }
    };
    f32x16 dq[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) dq[b] = zero16();
    f32x16 mean[NB];          // of the keys, and what the row's p (dp - delta) add up to: see above
    float rest = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) mean[b] = zero16();
    const float pos = (float)(i + see.shift - 4 * h);
    using Reader = TileReader<P>;
    const Reader reader(lane);
    auto compute = [&](int j0, uint32_t tile, bool masked) {       // tile: K's rows, V's behind them
        const uint32_t kr = tile + reader.rows, kc = tile + reader.columns;
        uint32_t gr = tile_address(parked) + 32 * wave * P * 2 + reader.rows;
        asm volatile("" : "+v"(gr));       // (not an address per step, kept all along the loop)
#pragma unroll
        for (int b = 0; b < STEP / 32; ++b) {
            f32x16 s = zero16(), dp = zero16();
            struct Rows {
                bf16x8 k, v, g;
            };
            __builtin_amdgcn_s_setprio(kMfmaPrio);
            read_ahead<NS, Rows>(
                [&](int k, Rows& r) {
                    r.k = Reader::frag(kr, 32 * b, k);
                    r.v = Reader::frag(kr, STEP + 32 * b, k);
                    if constexpr (PARKED) r.g = Reader::frag(gr, 0, k);
                    else r.g = gf[PARKED ? 0 : k];
                },
                [&](int k, const Rows& r) {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.k, qf[k], s, 0, 0, 0);
                    dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.v, r.g, dp, 0, 0, 0);
                });
            __builtin_amdgcn_s_setprio(0);
            f32x16 factor;
            const float away = pos - (float)j0;
            if constexpr (CAP) cap_scores(a.cap, rule.c, s);
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float p = s[v], g = dp[v] - delta;
                factor[v] = score_gradient<CAP, BIAS>(p, g, rule, offset, away - (float)(32 * b + acc_row(v)));
                s[v] = p;
                dp[v] = g;
            }
            if (masked) {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int j = j0 + 32 * b + acc_row(v) + 4 * h;
                    const bool seen = (j >= lo) & (j <= hi);
                    s[v] = seen ? s[v] : 0.f;
                    dp[v] = seen ? dp[v] : 0.f;
                }
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) rest += dp[v];
            if constexpr (CAP) {
                s *= factor;
                dp *= factor;
            }
            const bf16x8 df[2] = {score_frag(dp, 0), score_frag(dp, 1)}, pf[2] = {score_frag(s, 0), score_frag(s, 1)};
            __builtin_amdgcn_s_setprio(kMfmaPrio);
            read_ahead<2 * NB, bf16x8>([&](int n, bf16x8& k) { k = Reader::frag_t(kc, 32 * b + 16 * (n / NB), n % NB); },
                                            [&](int n, const bf16x8& k) {
                                                dq[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, df[n / NB], dq[n % NB], 0, 0, 0);
                                                mean[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, pf[n / NB], mean[n % NB], 0, 0, 0);
                                            });
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);     // (one block of scores at a time: more of them in flight spill)
        }
    };
    for (int step = begin; step < steps; ++step) {
        wait_loads<0>();
        lds_barrier();
        if (step + 1 < steps) fetch(step + 1, (step + 1) & 1);
        const int j0 = (first + step) * STEP;
        if (j0 > wave_hi || j0 + STEP <= wave_lo) continue;
        compute(j0, tile_address(smem) + (step & 1) * 4 * STEP * P, j0 < all_lo || j0 + STEP - 1 > all_hi);
    }
    rest += other_half(rest);
    if (a.parts > 1) {
        const int64_t row = ((int64_t)part * a.heads_q + head) * a.tokens_q + seq.q0 + i, rows = (int64_t)a.parts * a.heads_q * a.tokens_q;
        store_part(dq, a.part + row * a.d, a.d, mine, lane);
        store_part(mean, a.part + (rows + row) * a.d, a.d, mine, lane);
        if (mine && h == 0) a.part[2 * rows * a.d + row] = rest;
        if (part == 0) keep_stats(delta);
        return;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) dq[b][v] = __builtin_fmaf(-rest, mean[b][v], dq[b][v]);
    keep_stats(delta + rest);
    store_columns(dq, a.scale, a.dq + (int64_t)(seq.q0 + i) * a.dq_ts + (int64_t)head * a.dq_hs, a.d, mine, lane);
}

// Joins the parts of dq: four elements of a row per thread.
__global__ __launch_bounds__(256) void k_attention_dq_join(AttnArgs a) {
    const int per = a.d / 4;
    const int64_t rows = (int64_t)a.heads_q * a.tokens_q, at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / per;
    if (row >= rows) return;
    const int e = (int)(at - row * per) * 4, head = (int)(row / a.tokens_q), token = (int)(row - (int64_t)head * a.tokens_q);
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, mean = x;
    float rest = 0.f;
    for (int p = 0; p < a.parts; ++p) {
        const float* from = a.part + (rows * p + row) * a.d + e;
        x += *reinterpret_cast<const f32x4*>(from);
        mean += *reinterpret_cast<const f32x4*>(from + rows * a.parts * a.d);
        rest += a.part[2 * rows * a.parts * a.d + rows * p + row];
    }
    x = (x - mean * rest) * a.scale;
    if (e == 0) a.stats[rows + row] -= rest;
    const u32x2 w = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    *reinterpret_cast<u32x2*>(a.dq + (int64_t)token * a.dq_ts + (int64_t)head * a.dq_hs + e) = w;
}

// dk and dv: 128 keys per workgroup, 32 per wave; the queries of every head that shares them pass by, head after head.  Scores are [query][key] here, and
// their products begin at -delta and, where x is linear in the product, at lse's offset, which LDS holds for a step's queries.  V's rows are parked
// from d = 65 on, as dO's in dq.
template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_dkv(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16, STEP = attn_back_step<D>();
    constexpr bool PARKED = D > 64;
    constexpr int TILES = 4 * STEP * P + (PARKED ? kAttnRows * P : 0);
    // (one array: with two the compiler tells their loads apart, and waits again, for all in flight, ahead of the reads of each)
    __shared__ __attribute__((aligned(256))) uint16_t smem[TILES + 2 * 2 * 64 * 2];
    uint16_t* const parked = smem + 4 * STEP * P;
    float* const stats = reinterpret_cast<float*>(smem + TILES);       // [stage][offset of lse, -delta][64] of a step's queries
    const int heads_k = a.heads_q / a.group;
    int kv, t, part;
    if (!attn_place(heads_k, a.tiles, a.parts, kv, t, part)) return;
    const AttnTile seq = attn_tile<kAttnRows, true>(a, t);        // early tiles first: with a causal mask they have most queries
    const int row0 = seq.tile * kAttnRows;
    if (row0 < 0 || row0 >= seq.nk) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const int w0 = row0 + 32 * wave, j = w0 + (lane & 31);
    bf16x8 kf[NS], vf[PARKED ? 1 : NS];
    {
        const uint16_t* kp = a.k + (int64_t)(seq.k0 + row0) * a.k_ts + (int64_t)kv * a.k_hs;
        const uint16_t* vp = a.v + (int64_t)(seq.k0 + row0) * a.v_ts + (int64_t)kv * a.v_hs;
        const RowFrags kr(kp, a.k_ts, wave, lane, j < seq.nk, a.d), vr(vp, a.v_ts, wave, lane, j < seq.nk, a.d);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            kf[s] = kr.get(s);
            if constexpr (!PARKED) vf[s] = vr.get(s);
        }
        if constexpr (PARKED) {
            RowsTile<P, kAttnRows, 256> v;
            v.init(a.v_ts, a.d);
            v.load(parked, vp, a.v_ts, seq.nk - row0);
        }
    }
    // queries that see a key of the workgroup: causal, those from the key's position on (all, if the key lies in the prefix); with a
    // window, to the last one's position + window - 1
    const int end = min(row0 + kAttnRows, seq.nk) - 1;
    int qa = 0, qb = seq.nq;
    if (see.causal) {
        if (row0 >= see.prefix) qa = max(0, row0 - see.shift);
        if (see.window > 0) qb = (int)min((int64_t)qb, (int64_t)end - see.shift + see.window);
    }
    const int first = qa / STEP, steps = qb > qa ? (qb - 1) / STEP - first + 1 : 0, all = steps * a.group;
    int begin, total;
    attn_share(all, a.parts, part, begin, total);
    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) dk[b] = dv[b] = zero16();
    RowsTile<P, STEP, 256> qt, gt;
    qt.init(a.q_ts, a.d);
    gt.init(a.do_ts, a.d);
    // step `step` of the queries of head kv * group + `member`, in this order
    auto fetch = [&](int member, int step, int stage) {
        const int head = kv * a.group + member, i0 = (first + step) * STEP;
        qt.load(smem + stage * 2 * STEP * P, a.q + (int64_t)(seq.q0 + i0) * a.q_ts + (int64_t)head * a.q_hs, a.q_ts, seq.nq - i0);
        gt.load(smem + (stage * 2 + 1) * STEP * P, a.dO + (int64_t)(seq.q0 + i0) * a.do_ts + (int64_t)head * a.do_hs, a.do_ts, seq.nq - i0);
        // one array of statistics by half of the waves each; rows past the last are masked, and 0 is as good as any for them
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.stats + ((int64_t)(wave & 1) * a.heads_q + head) * a.tokens_q + seq.q0 + i0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(stats + (2 * stage + (wave & 1)) * 64), 4,
                                                 i0 + lane < seq.nq ? 4 * lane : 0x80000000u, 0, 0, 0);
    };
    // queries from .. to that see the lane's key
    const int from = see.causal && j >= see.prefix ? j - see.shift : 0;
    const int to = see.window > 0 ? min(seq.nq - 1, j - see.shift + see.window - 1) : seq.nq - 1;
    const float pos = (float)(j - see.shift - 4 * h);      // the distance from a register's query without its 4 h
    using Reader = TileReader<P>;
    const Reader reader(lane);
    auto compute = [&](int i0, uint32_t tile, uint32_t st, const ScoreRule& rule, bool masked) {       // tile: Q's rows, dO's behind them
        const uint32_t qr = tile + reader.rows, qc = tile + reader.columns;
        uint32_t vr = tile_address(parked) + 32 * wave * P * 2 + reader.rows;
        asm volatile("" : "+v"(vr));       // (not an address per step, kept all along the loop)
#pragma unroll
        for (int b = 0; b < STEP / 32; ++b) {
            f32x16 s, dp;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4 offset = lds_read4((lds_f32x4*)(st + (32 * b + 8 * r) * 4));
                const f32x4 delta = lds_read4((lds_f32x4*)(st + (64 + 32 * b + 8 * r) * 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[4 * r + e] = CAP || BIAS ? 0.f : offset[e];
                    dp[4 * r + e] = delta[e];
                }
            }
            struct Rows {
                bf16x8 q, g, v;
            };
            __builtin_amdgcn_s_setprio(kMfmaPrio);
            read_ahead<NS, Rows>(
                [&](int k, Rows& r) {
                    r.q = Reader::frag(qr, 32 * b, k);
                    r.g = Reader::frag(qr, STEP + 32 * b, k);
                    if constexpr (PARKED) r.v = Reader::frag(vr, 0, k);
                    else r.v = vf[PARKED ? 0 : k];
                },
                [&](int k, const Rows& r) {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.q, kf[k], s, 0, 0, 0);
                    dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.g, r.v, dp, 0, 0, 0);
                });
            __builtin_amdgcn_s_setprio(0);
            const float away = (float)i0 - pos;
            if constexpr (CAP) cap_scores(a.cap, rule.c, s);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                f32x4 offset = {0.f, 0.f, 0.f, 0.f};
                if constexpr (CAP || BIAS) offset = lds_read4((lds_f32x4*)(st + (32 * b + 8 * r) * 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p = s[4 * r + e], g = dp[4 * r + e];
                    const float factor = score_gradient<CAP, BIAS>(p, g, rule, offset[e], away + (float)(32 * b + 8 * r + e));
                    s[4 * r + e] = p;
                    dp[4 * r + e] = CAP ? g * factor : g;
                }
            }
            if (masked) {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int i = i0 + 32 * b + acc_row(v) + 4 * h;
                    const bool seen = (i >= from) & (i <= to);
                    s[v] = seen ? s[v] : 0.f;
                    dp[v] = seen ? dp[v] : 0.f;
                }
            }
            const bf16x8 pf[2] = {score_frag(s, 0), score_frag(s, 1)}, df[2] = {score_frag(dp, 0), score_frag(dp, 1)};
            struct Columns {
                bf16x8 g, q;
            };
            __builtin_amdgcn_s_setprio(kMfmaPrio);
            read_ahead<2 * NB, Columns>(
                [&](int n, Columns& r) {
                    r.g = Reader::frag_t(qc, STEP + 32 * b + 16 * (n / NB), n % NB);
                    r.q = Reader::frag_t(qc, 32 * b + 16 * (n / NB), n % NB);
                },
                [&](int n, const Columns& r) {
                    dv[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.g, pf[n / NB], dv[n % NB], 0, 0, 0);
                    dk[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(r.q, df[n / NB], dk[n % NB], 0, 0, 0);
                });
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int ahead = steps > 0 ? begin / steps : 0, ahead_step = begin - ahead * steps;       // what is fetched next: member and step
    auto fetch_next = [&](int it) {
        fetch(ahead, ahead_step, it & 1);
        if (++ahead_step == steps) {
            ahead_step = 0;
            ++ahead;
        }
    };
    int member = ahead, step = ahead_step;
    if (total > begin) fetch_next(begin);
    const int last_key = min(w0 + 31, seq.nk - 1);
    const uint32_t stats_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const float*)stats + 16 * h;
    for (int it = begin; it < total; ++it) {
        wait_loads<0>();
        lds_barrier();
        if (it + 1 < total) fetch_next(it + 1);
        const int now = kv * a.group + member, i0 = (first + step) * STEP, i1 = min(i0 + STEP, seq.nq) - 1;
        if (++step == steps) {
            step = 0;
            ++member;
        }
        if (w0 >= seq.nk || see.hi(i1) < w0 || see.lo(i0) > last_key) continue;
        const ScoreRule rule = score_rule<CAP, BIAS>(a, now);
        compute(i0, tile_address(smem) + (it & 1) * 4 * STEP * P, stats_at + (it & 1) * 2 * 64 * 4, rule, see.lo(i1) > w0 || see.hi(i0) < last_key || i0 + STEP > seq.nq);
    }
    const bool mine = j < seq.nk;
    if (a.parts > 1) {
        const int64_t rows = (int64_t)a.tokens_k * heads_k, row = (int64_t)(seq.k0 + j) * heads_k + kv;
        store_part(dk, a.part + (rows * (2 * part) + row) * a.d, a.d, mine, lane);
        store_part(dv, a.part + (rows * (2 * part + 1) + row) * a.d, a.d, mine, lane);
        return;
    }
    store_columns(dk, a.scale, a.dk + (int64_t)(seq.k0 + j) * a.dk_ts + (int64_t)kv * a.dk_hs, a.d, mine, lane);
    store_columns(dv, 1.f, a.dv + (int64_t)(seq.k0 + j) * a.dv_ts + (int64_t)kv * a.dv_hs, a.d, mine, lane);
}

// Joins the parts of dk and dv: four elements of both per thread.
__global__ __launch_bounds__(256) void k_attention_dkv_join(AttnArgs a) {
    const int per = a.d / 4, heads_k = a.heads_q / a.group;
    const int64_t rows = (int64_t)a.tokens_k * heads_k, at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / per;
    if (row >= rows) return;
    const int e = (int)(at - row * per) * 4, token = (int)(row / heads_k), kv = (int)(row - (int64_t)token * heads_k);
    f32x4 dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
    for (int p = 0; p < a.parts; ++p) {
        dk += *reinterpret_cast<const f32x4*>(a.part + (rows * (2 * p) + row) * a.d + e);
        dv += *reinterpret_cast<const f32x4*>(a.part + (rows * (2 * p + 1) + row) * a.d + e);
    }
    dk *= a.scale;
    const u32x2 wk = {pack_bf16x2(dk[0], dk[1]), pack_bf16x2(dk[2], dk[3])}, wv = {pack_bf16x2(dv[0], dv[1]), pack_bf16x2(dv[2], dv[3])};
    *reinterpret_cast<u32x2*>(a.dk + (int64_t)token * a.dk_ts + (int64_t)kv * a.dk_hs + e) = wk;
    *reinterpret_cast<u32x2*>(a.dv + (int64_t)token * a.dv_ts + (int64_t)kv * a.dv_hs + e) = wv;
}

// f(padded d, capped, biased) of a call's kernels: d in 64, 96 or 128.
template <typename F>
static void attn_shape(const qg_attention& a, F f) {
    using std::integral_constant;
    auto with_d = [&](auto cap, auto bias) {
        if (a.d <= 64) f(integral_constant<int, 64>(), cap, bias);
        else if (a.d <= 96) f(integral_constant<int, 96>(), cap, bias);
        else f(integral_constant<int, 128>(), cap, bias);
    };
    auto with_bias = [&](auto cap) { a.slopes != nullptr ? with_d(cap, std::true_type()) : with_d(cap, std::false_type()); };
    a.cap > 0.f ? with_bias(std::true_type()) : with_bias(std::false_type());
}

static int64_t attn_tiles(int64_t tokens, int sequences) { return tokens / kAttnRows + sequences + 1; }

static int check_attention(const qg_attention* a) {
    if (a == nullptr) return QG_ERR_NULL;
    if ((a->sequences != 1 && a->cu_q == nullptr) || ((a->cu_k != nullptr) && a->cu_q == nullptr)) return QG_ERR_NULL;
    if (a->tokens_q <= 0 || a->tokens_k <= 0 || a->tokens_q >= kAttnMaxTokens || a->tokens_k >= kAttnMaxTokens) return QG_ERR_SHAPE;
    if (a->heads_q <= 0 || a->heads_k <= 0 || a->heads_q % a->heads_k != 0 || a->heads_q > kAttnMaxHeads) return QG_ERR_SHAPE;
    if (a->d <= 0 || a->d > 128 || a->d % 8 != 0 || a->sequences <= 0 || a->sequences > kAttnMaxSequences) return QG_ERR_SHAPE;
    if (a->cu_k == nullptr && a->cu_q != nullptr && a->tokens_q != a->tokens_k) return QG_ERR_SHAPE;
    if (!check_scores(a->scale, a->cap)) return QG_ERR_SHAPE;
    if (a->window < 0 || (!a->causal && (a->window > 0 || a->prefix != nullptr)) || (a->window > 0 && a->prefix != nullptr)) return QG_ERR_SHAPE;
    for (const void* p : {(const void*)a->cu_q, (const void*)a->cu_k, (const void*)a->prefix, (const void*)a->slopes})
        if (reinterpret_cast<uintptr_t>(p) & 3) return QG_ERR_ALIGN;
    // fewer than 2^32 threads in a launch
    const int64_t most = (attn_tiles(a->tokens_q > a->tokens_k ? a->tokens_q : a->tokens_k, a->sequences)) * a->heads_q;
    if (most * 256 >= (int64_t(1) << 32) - 4096) return QG_ERR_SHAPE;
    return QG_OK;
}

int check_heads(const qg_heads* x, bool required, int unit) {
    if (x == nullptr || x->data == nullptr) return required ? QG_ERR_NULL : QG_OK;
    if (reinterpret_cast<uintptr_t>(x->data) % (2 * unit)) return QG_ERR_ALIGN;
    if (x->token_stride < 0 || x->head_stride < 0 || x->token_stride >= kHeadsMaxStride || x->head_stride >= (int64_t(1) << 40)) return QG_ERR_SHAPE;
    return (x->token_stride | x->head_stride) % unit ? QG_ERR_ALIGN : QG_OK;
}

static AttnArgs attn_args(const qg_attention* a, const qg_heads* q, const qg_heads* k, const qg_heads* v, const qg_heads* o, float* lse) {
    AttnArgs r = {};
    r.q = q->data, r.q_ts = q->token_stride, r.q_hs = q->head_stride;
    r.k = k->data, r.k_ts = k->token_stride, r.k_hs = k->head_stride;
    r.v = v->data, r.v_ts = v->token_stride, r.v_hs = v->head_stride;
    r.o = o->data, r.o_ts = o->token_stride, r.o_hs = o->head_stride;
    r.lse = lse;
    r.cu_q = a->cu_q;
    r.cu_k = a->cu_k != nullptr ? a->cu_k : a->cu_q;
    r.prefix = a->prefix, r.slopes = a->slopes;
    r.tokens_q = (int)a->tokens_q, r.tokens_k = (int)a->tokens_k;
    r.heads_q = a->heads_q, r.group = a->heads_q / a->heads_k, r.d = a->d, r.sequences = a->sequences;
    r.causal = a->causal != 0;
    r.window = (int)(a->window < kAttnMaxTokens * 2 ? a->window : 0);   // (a window beyond every sequence is none)
    r.scale = a->scale, r.cap = a->cap;
    return r;
}

// Workgroups of `tiles` tiles of rows, `heads` of them and parts.
static dim3 attn_grid(const AttnArgs& a, int heads) { return dim3((unsigned)(((int64_t)a.tiles * heads * a.parts + 7) / 8 * 8)); }
static dim3 join_grid(int64_t rows, int d) { return dim3((unsigned)((rows * (d / 4) + 255) / 256)); }

// Parts of the keys of a call with few tiles of queries (forward, dq), and of the queries, of all heads that share a key head, of one with few
// tiles of keys (dkv); their fp32 sums go through the workspace and are joined in order.  `steps`: of 64 rows, of a sequence in the mean.
struct AttnParts {
    int forward, dq, dkv;
};
static int attn_parts(int64_t parts, int64_t steps, int least) {
    const int64_t most = steps / least;     // (a part of fewer steps costs more in its ends and in the join than it saves)
    return (int)(parts < 1 || most < 1 ? 1 : parts < most ? (parts < 16 ? parts : 16) : most < 16 ? most : 16);
}
// Keys: whole parts of 512 workgroups (us without / with; 2048 queries, 8 heads of 128 on one key head: forward 41 / 31; 4096, one head of 64: 56 / 22,
// backward 196 / 70; but 2000, 24 heads, 432 tiles, in two parts: 27 / 34).  Queries: 1024 workgroups or more, since a causal mask gives
// the first keys most of the work (us in one part / by the rule / for 2048: 8192 tokens, 32 heads on 8 of 128: backward 3140 / 2270 / 2230; 4096, 16 on
// 4, four sequences: 343 / 184 / 207; 4096, 32 on 32 without a mask, 1088 tiles: 1092 / 1091 / 1225), of 16 steps or more (backward with four / 16 / 24: 8 sequences
// of 512, 12 heads of 64: 58 / 39 / -; 4 of 1024, 16 of 64: 86 / 67 / 67; 16 on 4 of 128: 145 / 134 / 164); of two where the
// parts are few all the same (2000, 4 on 1, ten sequences: 32 / 29).
static AttnParts attn_parts(const qg_attention* a) {
    const int64_t work_q = attn_tiles(a->tokens_q, a->sequences) * a->heads_q, work_k = attn_tiles(a->tokens_k, a->sequences) * a->heads_k;
    const int keys = attn_parts(512 / work_q, a->tokens_k / a->sequences / 64, 4);
    return {keys, keys, attn_parts((1024 + work_k - 1) / work_k, a->tokens_q / a->sequences * (a->heads_q / a->heads_k) / 64, work_k < 128 ? 2 : 16)};
}
// Floats of the parts' sums.
static int64_t forward_floats(const qg_attention* a, int parts) { return parts > 1 ? (int64_t)parts * a->heads_q * a->tokens_q * (a->d + 2) : 0; }
static int64_t backward_floats(const qg_attention* a, const AttnParts& p) {
    const int64_t dq = p.dq > 1 ? (int64_t)p.dq * a->heads_q * a->tokens_q * (2 * a->d + 1) : 0;
    const int64_t dkv = p.dkv > 1 ? (int64_t)p.dkv * a->heads_k * a->tokens_k * 2 * a->d : 0;
    return dq > dkv ? dq : dkv;
}
static int64_t stats_floats(const qg_attention* a) { return ((int64_t)a->heads_q * a->tokens_q * 2 + 3) / 4 * 4; }

}  // namespace qg

using namespace qg;

extern "C" size_t qg_attention_forward_workspace_bytes(const qg_attention* a) {
    return check_attention(a) == QG_OK ? (size_t)forward_floats(a, attn_parts(a).forward) * 4 : 0;
}

extern "C" size_t qg_attention_backward_workspace_bytes(const qg_attention* a) {
    return check_attention(a) == QG_OK ? (size_t)(stats_floats(a) + backward_floats(a, attn_parts(a))) * 4 : 0;
}

extern "C" int qg_attention_forward(const qg_attention* a, const qg_heads* q, const qg_heads* k, const qg_heads* v, const qg_heads* o,
                                    float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (int e = check_attention(a)) return e;
    for (const qg_heads* x : {q, k, v, o})
        if (int e = check_heads(x, true)) return e;
    if ((reinterpret_cast<uintptr_t>(lse) & 3) || !aligned16(workspace)) return QG_ERR_ALIGN;
    AttnArgs args = attn_args(a, q, k, v, o, lse);
    args.parts = attn_parts(a).forward;
    const size_t need = (size_t)forward_floats(a, args.parts) * 4;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return QG_ERR_WORKSPACE;
    args.part = static_cast<float*>(workspace);
    args.tiles = (int)attn_tiles(a->tokens_q, a->sequences);
    attn_shape(*a, [&](auto d, auto cap, auto bias) {
        hipLaunchKernelGGL((k_attention_fwd<d.value, cap.value, bias.value>), attn_grid(args, args.heads_q), dim3(256), 0, (hipStream_t)stream, args);
    });
    if (args.parts > 1)
        hipLaunchKernelGGL(k_attention_fwd_join, join_grid(a->tokens_q * a->heads_q, a->d), dim3(256), 0, (hipStream_t)stream, args);
    return check_launch();
}

extern "C" int qg_attention_backward(const qg_attention* a, const qg_heads* dO, const qg_heads* q, const qg_heads* k, const qg_heads* v,
                                     const qg_heads* o, const float* lse, const qg_heads* dq, const qg_heads* dk, const qg_heads* dv,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    if (int e = check_attention(a)) return e;
    for (const qg_heads* x : {dO, q, k, v, o, dq, dk, dv})
        if (int e = check_heads(x, true)) return e;
    if (lse == nullptr) return QG_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(lse) & 3) || !aligned16(workspace)) return QG_ERR_ALIGN;
    if (workspace == nullptr || workspace_bytes < qg_attention_backward_workspace_bytes(a)) return QG_ERR_WORKSPACE;
    AttnArgs args = attn_args(a, q, k, v, o, const_cast<float*>(lse));
    args.dO = dO->data, args.do_ts = dO->token_stride, args.do_hs = dO->head_stride;
    args.dq = dq->data, args.dq_ts = dq->token_stride, args.dq_hs = dq->head_stride;
    args.dk = dk->data, args.dk_ts = dk->token_stride, args.dk_hs = dk->head_stride;
    args.dv = dv->data, args.dv_ts = dv->token_stride, args.dv_hs = dv->head_stride;
    args.stats = static_cast<float*>(workspace);
    args.part = args.stats + stats_floats(a);
    const AttnParts parts = attn_parts(a);
    attn_shape(*a, [&](auto d, auto cap, auto bias) {
        args.tiles = (int)attn_tiles(a->tokens_q, a->sequences), args.parts = parts.dq;
        hipLaunchKernelGGL((k_attention_dq<d.value, cap.value, bias.value>), attn_grid(args, a->heads_q), dim3(256), 0, (hipStream_t)stream, args);
        if (parts.dq > 1)
            hipLaunchKernelGGL(k_attention_dq_join, join_grid(a->tokens_q * a->heads_q, a->d), dim3(256), 0, (hipStream_t)stream, args);
        args.tiles = (int)attn_tiles(a->tokens_k, a->sequences), args.parts = parts.dkv;
        hipLaunchKernelGGL((k_attention_dkv<d.value, cap.value, bias.value>), attn_grid(args, a->heads_k), dim3(256), 0, (hipStream_t)stream, args);
        if (parts.dkv > 1)
            hipLaunchKernelGGL(k_attention_dkv_join, join_grid(a->tokens_k * a->heads_k, a->d), dim3(256), 0, (hipStream_t)stream, args);
    });
    return check_launch();
}
