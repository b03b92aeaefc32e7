// Attention over packed sequences, forward and backward.  With x = scale q.k, capped cap tanh(x / cap), minus slope |distance|, over the
// visible keys of a query (qg_attention.h):
//     lse = log sum_j exp(x_j),   p_j = exp(x_j - lse),   o = sum_j p_j v_j
//     delta = sum_d do o,   ds_j = p_j (do.v_j - delta) (1 - tanh^2) scale
//     dq = sum_j ds_j k_j,   dk_j = sum_i ds_ij q_i,   dv_j = sum_i p_ij do_i
// One pass over the keys with a running maximum and sum; exponentials to the base 2.  p and ds are rounded to bf16, operands of
// matrix products, as every product of the library has them; maxima, sums, lse, delta and all accumulators are fp32.
// Backward: one kernel for dq (queries stay, keys pass by) and one for dk and dv (keys stay, queries of all heads that share them
// pass by): seven products where one kernel would do five, but each sum has one owner and one order: no atomics, the same bits every time.
#include "qg_attention.h"

namespace qg {

constexpr int kAttnWaves = 4;      // of a workgroup, 32 rows each
constexpr int kAttnRows = 32 * kAttnWaves;
constexpr int kAttnStep = 64;      // rows that pass by, per step

template <int D>
constexpr int attn_pitch() { return D <= 64 ? 64 : 128; }

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
        prefix = a.prefix != nullptr && t.seq < a.sequences ? a.prefix[t.seq] : 0;
        window = a.window;
    }
    __device__ __forceinline__ int hi(int i) const { return causal ? min(last, max(i + shift, prefix - 1)) : last; }
    __device__ __forceinline__ int lo(int i) const { return window > 0 ? max(0, i + shift - window + 1) : 0; }
};

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_fwd(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16;
    __shared__ __attribute__((aligned(16))) uint16_t smem[4 * kAttnStep * P];
    int head, t;
    if (!attn_place(a.heads_q * a.tiles, a.tiles, head, t)) return;
    const AttnTile seq = attn_tile<kAttnRows, false>(a, a.tiles - 1 - t);   // late tiles first: with a causal mask they have most keys
    const int row0 = seq.tile * kAttnRows;
    if (row0 >= seq.nq) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const ScoreRule rule = score_rule<CAP, BIAS>(a, head);
    const int kv = head / a.group;
    const uint16_t* qp = a.q + (int64_t)seq.q0 * a.q_ts + (int64_t)head * a.q_hs;
    const uint16_t* kp = a.k + (int64_t)seq.k0 * a.k_ts + (int64_t)kv * a.k_hs;
    const uint16_t* vp = a.v + (int64_t)seq.k0 * a.v_ts + (int64_t)kv * a.v_hs;

    const int w0 = row0 + 32 * wave, i = w0 + (lane & 31), w1 = min(w0 + 31, seq.nq - 1);
    bf16x8 qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = row_frag(qp, a.q_ts, i, seq.nq, s, a.d, lane);
    const int lo = see.lo(i), hi = see.hi(i);
    // steps that some row of the workgroup sees, and, of the wave, those that all rows see whole
    const int first = see.lo(row0) / kAttnStep, last = see.hi(min(row0 + kAttnRows, seq.nq) - 1) / kAttnStep;
    const int steps = see.hi(min(row0 + kAttnRows, seq.nq) - 1) < 0 ? 0 : last - first + 1;
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
    const float pos = (float)(i + see.shift);
    auto compute = [&](int j0, const uint16_t* K, const uint16_t* V, auto masked) {
        f32x16 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            s[b] = zero16();
#pragma unroll
            for (int k = 0; k < NS; ++k) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag<P>(K, 32 * b, k, lane), qf[k], s[b], 0, 0, 0);
        }
        constexpr bool kScaled = CAP || BIAS;     // s already holds x log2(e)
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int j = j0 + 32 * b + acc_row(v) + 4 * h;
                if constexpr (kScaled) {
                    float unused;
                    s[b][v] = score_log2<CAP>(s[b][v], rule.c, rule.cap_log2e, unused);
                    if constexpr (BIAS) s[b][v] = __builtin_fmaf(-rule.slope, fabsf(pos - (float)j), s[b][v]);
                }
                if constexpr (decltype(masked)::value) s[b][v] = j >= lo && j <= hi ? s[b][v] : -INFINITY;
                top = fmaxf(top, s[b][v]);
            }
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
                    o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag_t<P>(V, 32 * b + 16 * u, c, lane), pf, o[c], 0, 0, 0);
            }
    };

    if (steps > 0) fetch(0, 0);
    for (int step = 0; step < steps; ++step) {
        wait_loads<0>();
        lds_barrier();
        if (step + 1 < steps) fetch(step + 1, (step + 1) & 1);
        const int j0 = (first + step) * kAttnStep;
        const uint16_t *K = smem + (step & 1) * 2 * kAttnStep * P, *V = K + kAttnStep * P;
        if (j0 > wave_hi || j0 + kAttnStep <= wave_lo) continue;
        if (j0 >= all_lo && j0 + kAttnStep - 1 <= all_hi) compute(j0, K, V, std::false_type());
        else compute(j0, K, V, std::true_type());
    }
    l += other_half(l);
    const bool mine = i < seq.nq;
    if (mine && h == 0 && a.lse != nullptr)
        a.lse[(int64_t)head * a.tokens_q + seq.q0 + i] = l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    store_columns(o, l == 0.f ? 0.f : 1.f / l, a.o + (int64_t)(seq.q0 + i) * a.o_ts + (int64_t)head * a.o_hs, a.d, mine, lane);
}

// The scores' gradients of one 32 x 32 block, from the products s and dp (in place: s becomes p, dp becomes ds / scale).
// lse2, delta: per register or per lane; the position and the visible interval too.
template <bool CAP, bool BIAS, bool MASKED>
__device__ __forceinline__ void score_gradient(float& s, float& dp, const ScoreRule& rule, float lse2, float delta, int j, float pos, int lo, int hi) {
    float factor;
    float x = score_log2<CAP>(s, rule.c, rule.cap_log2e, factor);
    if constexpr (BIAS) x = __builtin_fmaf(-rule.slope, fabsf(pos - (float)j), x);
    const bool seen = !MASKED || (j >= lo && j <= hi);
    float p = __builtin_amdgcn_exp2f(x - lse2);
    float g = p * (dp - delta);
    if constexpr (CAP) g *= factor;
    s = seen ? p : 0.f;
    dp = seen ? g : 0.f;
}

// lse as the exponent's offset: a row without a visible key has p = 0.
__device__ __forceinline__ float lse_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_attention_dq(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16;
    __shared__ __attribute__((aligned(16))) uint16_t smem[4 * kAttnStep * P];
    int head, t;
    if (!attn_place(a.heads_q * a.tiles, a.tiles, head, t)) return;
    const AttnTile seq = attn_tile<kAttnRows, false>(a, a.tiles - 1 - t);
    const int row0 = seq.tile * kAttnRows;
    if (row0 >= seq.nq) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const ScoreRule rule = score_rule<CAP, BIAS>(a, head);
    const int kv = head / a.group;
    const uint16_t* kp = a.k + (int64_t)seq.k0 * a.k_ts + (int64_t)kv * a.k_hs;
    const uint16_t* vp = a.v + (int64_t)seq.k0 * a.v_ts + (int64_t)kv * a.v_hs;
    const int w0 = row0 + 32 * wave, i = w0 + (lane & 31), w1 = min(w0 + 31, seq.nq - 1);
    const bool mine = i < seq.nq;
    bf16x8 qf[NS], gf[NS];
    float delta = 0.f;
    {
        const uint16_t* qp = a.q + (int64_t)seq.q0 * a.q_ts + (int64_t)head * a.q_hs;
        const uint16_t* gp = a.dO + (int64_t)seq.q0 * a.do_ts + (int64_t)head * a.do_hs;
        const uint16_t* op = a.o + (int64_t)seq.q0 * a.o_ts + (int64_t)head * a.o_hs;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            qf[s] = row_frag(qp, a.q_ts, i, seq.nq, s, a.d, lane);
            gf[s] = row_frag(gp, a.do_ts, i, seq.nq, s, a.d, lane);
            const bf16x8 of = row_frag(op, a.o_ts, i, seq.nq, s, a.d, lane);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)gf[s][e], (float)of[e], delta);
        }
        delta += other_half(delta);
    }
    const int64_t at = (int64_t)head * a.tokens_q + seq.q0 + i;
    if (mine && h == 0) a.delta[at] = delta;
    const float lse2 = mine ? lse_log2(a.lse[at]) : INFINITY;
    const int lo = see.lo(i), hi = see.hi(i);
    const int first = see.lo(row0) / kAttnStep, most = see.hi(min(row0 + kAttnRows, seq.nq) - 1);
    const int steps = most < 0 ? 0 : most / kAttnStep - first + 1;
    const int wave_lo = see.lo(w0), wave_hi = w0 < seq.nq ? see.hi(w1) : -1, all_lo = see.lo(w1), all_hi = see.hi(w0);
    f32x16 dq[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) dq[b] = zero16();
    RowsTile<P, kAttnStep, 256> kt, vt;
    kt.init(a.k_ts, a.d);
    vt.init(a.v_ts, a.d);
    auto fetch = [&](int step, int stage) {
        const int j = (first + step) * kAttnStep;
        kt.load(smem + stage * 2 * kAttnStep * P, kp + (int64_t)j * a.k_ts, a.k_ts, seq.nk - j);
        vt.load(smem + (stage * 2 + 1) * kAttnStep * P, vp + (int64_t)j * a.v_ts, a.v_ts, seq.nk - j);
    };
    const float pos = (float)(i + see.shift);
    auto compute = [&](int j0, const uint16_t* K, const uint16_t* V, auto masked) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int k = 0; k < NS; ++k) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag<P>(K, 32 * b, k, lane), qf[k], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag<P>(V, 32 * b, k, lane), gf[k], dp, 0, 0, 0);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                float p = s[v], g = dp[v];
                score_gradient<CAP, BIAS, decltype(masked)::value>(p, g, rule, lse2, delta, j0 + 32 * b + acc_row(v) + 4 * h, pos, lo, hi);
                dp[v] = g;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 df = score_frag(dp, u);
#pragma unroll
                for (int c = 0; c < NB; ++c)
                    dq[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag_t<P>(K, 32 * b + 16 * u, c, lane), df, dq[c], 0, 0, 0);
            }
        }
    };
    if (steps > 0) fetch(0, 0);
    for (int step = 0; step < steps; ++step) {
        wait_loads<0>();
        lds_barrier();
        if (step + 1 < steps) fetch(step + 1, (step + 1) & 1);
        const int j0 = (first + step) * kAttnStep;
        const uint16_t *K = smem + (step & 1) * 2 * kAttnStep * P, *V = K + kAttnStep * P;
        if (j0 > wave_hi || j0 + kAttnStep <= wave_lo) continue;
        if (j0 >= all_lo && j0 + kAttnStep - 1 <= all_hi) compute(j0, K, V, std::false_type());
        else compute(j0, K, V, std::true_type());
    }
    store_columns(dq, a.scale, a.dq + (int64_t)(seq.q0 + i) * a.dq_ts + (int64_t)head * a.dq_hs, a.d, mine, lane);
}

template <int D, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 1) void k_attention_dkv(AttnArgs a) {
    constexpr int P = attn_pitch<D>(), NB = D / 32, NS = D / 16;
    __shared__ __attribute__((aligned(16))) uint16_t smem[4 * kAttnStep * P];
    __shared__ __attribute__((aligned(16))) float stats[2][2][kAttnStep];   // lse and delta of a step's queries
    const int heads_k = a.heads_q / a.group;
    int kv, t;
    if (!attn_place(heads_k * a.tiles, a.tiles, kv, t)) return;
    const AttnTile seq = attn_tile<kAttnRows, true>(a, t);        // early tiles first: with a causal mask they have most queries
    const int row0 = seq.tile * kAttnRows;
    if (row0 >= seq.nk) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const Visible see(a, seq);
    const int w0 = row0 + 32 * wave, j = w0 + (lane & 31);
    bf16x8 kf[NS], vf[NS];
    {
        const uint16_t* kp = a.k + (int64_t)seq.k0 * a.k_ts + (int64_t)kv * a.k_hs;
        const uint16_t* vp = a.v + (int64_t)seq.k0 * a.v_ts + (int64_t)kv * a.v_hs;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            kf[s] = row_frag(kp, a.k_ts, j, seq.nk, s, a.d, lane);
            vf[s] = row_frag(vp, a.v_ts, j, seq.nk, s, a.d, lane);
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
    const int first = qa / kAttnStep, steps = qb > qa ? (qb - 1) / kAttnStep - first + 1 : 0, total = steps * a.group;
    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) dk[b] = dv[b] = zero16();
    RowsTile<P, kAttnStep, 256> qt, gt;
    qt.init(a.q_ts, a.d);
    gt.init(a.do_ts, a.d);
    auto fetch = [&](int it, int stage) {
        const int head = kv * a.group + it / steps, i0 = (first + it % steps) * kAttnStep;
        qt.load(smem + stage * 2 * kAttnStep * P, a.q + (int64_t)(seq.q0 + i0) * a.q_ts + (int64_t)head * a.q_hs, a.q_ts, seq.nq - i0);
        gt.load(smem + (stage * 2 + 1) * kAttnStep * P, a.dO + (int64_t)(seq.q0 + i0) * a.do_ts + (int64_t)head * a.do_hs, a.do_ts, seq.nq - i0);
    };
    // lse and delta of a step: read into registers a step ahead, put into LDS with the barrier
    float stat = 0.f;
    auto fetch_stats = [&](int it) {
        const int head = kv * a.group + it / steps, i = (first + it % steps) * kAttnStep + (threadIdx.x & 63);
        const int64_t at = (int64_t)head * a.tokens_q + seq.q0 + i;
        if (threadIdx.x < 64) stat = i < seq.nq ? lse_log2(a.lse[at]) : INFINITY;
        else if (threadIdx.x < 128) stat = i < seq.nq ? a.delta[at] : 0.f;
    };
    auto compute = [&](int i0, const uint16_t* Q, const uint16_t* G, const float (*st)[kAttnStep], const ScoreRule& rule, auto masked) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int k = 0; k < NS; ++k) {
                s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag<P>(Q, 32 * b, k, lane), kf[k], s, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag<P>(G, 32 * b, k, lane), vf[k], dp, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const f32x4 lse2 = *reinterpret_cast<const f32x4*>(&st[0][32 * b + 8 * r + 4 * h]);
                const f32x4 delta = *reinterpret_cast<const f32x4*>(&st[1][32 * b + 8 * r + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = i0 + 32 * b + 8 * r + 4 * h + e;
                    float p = s[4 * r + e], g = dp[4 * r + e];
                    int lo = 0, hi = 0;
                    if constexpr (decltype(masked)::value) {
                        lo = see.lo(i);
                        hi = see.hi(i);
                    }
                    score_gradient<CAP, BIAS, decltype(masked)::value>(p, g, rule, lse2[e], delta[e], j, (float)(i + see.shift), lo, hi);
                    s[4 * r + e] = p;
                    dp[4 * r + e] = g;
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bf16x8 pf = score_frag(s, u), df = score_frag(dp, u);
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    dv[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag_t<P>(G, 32 * b + 16 * u, c, lane), pf, dv[c], 0, 0, 0);
                    dk[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_frag_t<P>(Q, 32 * b + 16 * u, c, lane), df, dk[c], 0, 0, 0);
                }
            }
        }
    };
    if (total > 0) {
        fetch(0, 0);
        fetch_stats(0);
    }
    const int last_key = min(w0 + 31, seq.nk - 1);
    for (int it = 0; it < total; ++it) {
        wait_loads<0>();
        if (threadIdx.x < 128) stats[it & 1][threadIdx.x >> 6][threadIdx.x & 63] = stat;
        lds_barrier();
        if (it + 1 < total) {
            fetch(it + 1, (it + 1) & 1);
            fetch_stats(it + 1);
        }
        const int i0 = (first + it % steps) * kAttnStep, i1 = min(i0 + kAttnStep, seq.nq) - 1;
        const uint16_t *Q = smem + (it & 1) * 2 * kAttnStep * P, *G = Q + kAttnStep * P;
        if (w0 >= seq.nk || see.hi(i1) < w0 || see.lo(i0) > last_key) continue;
        const ScoreRule rule = score_rule<CAP, BIAS>(a, kv * a.group + it / steps);
        if (see.lo(i1) <= w0 && see.hi(i0) >= last_key) compute(i0, Q, G, stats[it & 1], rule, std::false_type());
        else compute(i0, Q, G, stats[it & 1], rule, std::true_type());
    }
    const bool mine = j < seq.nk;
    store_columns(dk, a.scale, a.dk + (int64_t)(seq.k0 + j) * a.dk_ts + (int64_t)kv * a.dk_hs, a.d, mine, lane);
    store_columns(dv, 1.f, a.dv + (int64_t)(seq.k0 + j) * a.dv_ts + (int64_t)kv * a.dv_hs, a.d, mine, lane);
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
    if (!(a->scale > 0.f && a->scale < INFINITY) || !(a->cap >= 0.f && a->cap < INFINITY)) return QG_ERR_SHAPE;
    if (a->window < 0 || (!a->causal && (a->window > 0 || a->prefix != nullptr)) || (a->window > 0 && a->prefix != nullptr)) return QG_ERR_SHAPE;
    for (const void* p : {(const void*)a->cu_q, (const void*)a->cu_k, (const void*)a->prefix, (const void*)a->slopes})
        if (reinterpret_cast<uintptr_t>(p) & 3) return QG_ERR_ALIGN;
    // fewer than 2^32 threads in a launch
    const int64_t most = (attn_tiles(a->tokens_q > a->tokens_k ? a->tokens_q : a->tokens_k, a->sequences)) * a->heads_q;
    if (most * 256 >= (int64_t(1) << 32) - 4096) return QG_ERR_SHAPE;
    return QG_OK;
}

int check_heads(const qg_heads* x, bool required) {
    if (x == nullptr || x->data == nullptr) return required ? QG_ERR_NULL : QG_OK;
    if (!aligned16(x->data)) return QG_ERR_ALIGN;
    if (x->token_stride < 0 || x->head_stride < 0 || x->token_stride >= kHeadsMaxStride || x->head_stride >= (int64_t(1) << 40)) return QG_ERR_SHAPE;
    return ((x->token_stride | x->head_stride) & 7) ? QG_ERR_ALIGN : QG_OK;
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

static dim3 attn_grid(int64_t work) { return dim3((unsigned)((work + 7) / 8 * 8)); }

}  // namespace qg

using namespace qg;

extern "C" size_t qg_attention_workspace_bytes(const qg_attention* a) {
    if (check_attention(a) != QG_OK) return 0;
    return ((size_t)a->heads_q * a->tokens_q * 4 + 15) / 16 * 16;
}

extern "C" int qg_attention_forward(const qg_attention* a, const qg_heads* q, const qg_heads* k, const qg_heads* v, const qg_heads* o,
                                    float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    (void)workspace, (void)workspace_bytes;
    if (int e = check_attention(a)) return e;
    for (const qg_heads* x : {q, k, v, o})
        if (int e = check_heads(x, true)) return e;
    if (reinterpret_cast<uintptr_t>(lse) & 3) return QG_ERR_ALIGN;
    AttnArgs args = attn_args(a, q, k, v, o, lse);
    args.tiles = (int)attn_tiles(a->tokens_q, a->sequences);
    attn_shape(*a, [&](auto d, auto cap, auto bias) {
        hipLaunchKernelGGL((k_attention_fwd<d.value, cap.value, bias.value>), attn_grid((int64_t)args.tiles * args.heads_q), dim3(256), 0,
                           (hipStream_t)stream, args);
    });
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
    if (workspace == nullptr || workspace_bytes < qg_attention_workspace_bytes(a)) return QG_ERR_WORKSPACE;
    AttnArgs args = attn_args(a, q, k, v, o, const_cast<float*>(lse));
    args.dO = dO->data, args.do_ts = dO->token_stride, args.do_hs = dO->head_stride;
    args.dq = dq->data, args.dq_ts = dq->token_stride, args.dq_hs = dq->head_stride;
    args.dk = dk->data, args.dk_ts = dk->token_stride, args.dk_hs = dk->head_stride;
    args.dv = dv->data, args.dv_ts = dv->token_stride, args.dv_hs = dv->head_stride;
    args.delta = static_cast<float*>(workspace);
    attn_shape(*a, [&](auto d, auto cap, auto bias) {
        args.tiles = (int)attn_tiles(a->tokens_q, a->sequences);
        hipLaunchKernelGGL((k_attention_dq<d.value, cap.value, bias.value>), attn_grid((int64_t)args.tiles * args.heads_q), dim3(256), 0,
                           (hipStream_t)stream, args);
        args.tiles = (int)attn_tiles(a->tokens_k, a->sequences);
        hipLaunchKernelGGL((k_attention_dkv<d.value, cap.value, bias.value>), attn_grid((int64_t)args.tiles * a->heads_k), dim3(256), 0,
                           (hipStream_t)stream, args);
    });
    return check_launch();
}
