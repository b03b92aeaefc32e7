// Rotary positions of q and k, and their way into a cache of pages.  A pair (a, b) of a head becomes
//     amplitude (a cos t - b sin t, a sin t + b cos t),  t = position * frequency;  the backward pass turns by -t.
// The angle is formed and reduced to one turn in 64 bits (a far position times a frequency loses it in 32), its sine and cosine are fp32, and
// the result is rounded once.  A workgroup computes the sines of its tokens once, for all heads, into LDS; then every element
// is read and written once: HBM is the bound (4096 tokens, 32 + 32 heads of 128: 24.6 us, 5.5 TB/s with part of the inputs in the last-level cache;
// 4000 tokens into a cache, 32 + 8 heads: 17.7 us), for a few tokens the chain of position, frequency and sine ahead of the first store (2.8 us).
#include "qg_attention.h"

#include <cmath>

namespace qg {

constexpr int kRopeMaxD = 1024, kRopeTable = 2048;   // (sine, cosine) pairs of a workgroup's tokens

struct RopeStream {      // one of q, k, v: `heads` heads of d elements per token
    const uint16_t* src;
    uint16_t* dst;
    int64_t src_ts, src_hs, dst_ts, dst_hs;
    int heads, turned, copied;   // pieces of a head that are turned, and those that are only copied (none in place)
    bool paged;                  // dst is a cache: dst_ts is the distance of its rows, dst_hs of its heads
};

struct RopeArgs {
    RopeStream s[3];
    const int64_t* positions;
    const double* freqs;
    int64_t tokens;
    int d, rot, tokens_per_group, items;   // items: pieces of a token in all streams
    float amplitude, sign;
    // the cache
    const int32_t *table, *sequence;
    int64_t pages;
    int page_size, sequences, width;
};

// One piece of a head: INTERLEAVED: the turned elements 8 c .. 8 c + 7 (4 pairs); else pairs 8 c .. 8 c + 7 of the halves.  Piece `turned` and on: 8 of
// the elements from rot on.
template <bool INTERLEAVED>
__device__ __forceinline__ void rope_piece(const RopeArgs& a, const RopeStream& s, const uint16_t* src, uint16_t* dst, int c, const float2* turn) {
    if (c >= s.turned) {
        const int at = (s.turned ? a.rot : 0) + 8 * (c - s.turned), n = min(8, a.d - at);
        if (n == 8) {
            *reinterpret_cast<u32x4_align2*>(dst + at) = *reinterpret_cast<const u32x4_align2*>(src + at);
        } else {
            for (int e = 0; e < n; ++e) dst[at + e] = src[at + e];
        }
        return;
    }
    auto value = [](uint32_t w, int e) { return __builtin_bit_cast(float, e ? w & 0xFFFF0000u : w << 16); };
    auto round2 = [](const float2 cs, float x, float y, float& u, float& v) {
        u = __builtin_fmaf(x, cs.x, -(y * cs.y));
        v = __builtin_fmaf(x, cs.y, y * cs.x);
    };
    if constexpr (INTERLEAVED) {
        const int at = 8 * c, n = min(8, a.rot - at);
        const float2* t = turn + at / 2;
        if (n == 8) {
            u32x4 w = *reinterpret_cast<const u32x4_align2*>(src + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float u, v;
                round2(t[e], value(w[e], 0), value(w[e], 1), u, v);
                w[e] = pack_bf16x2(u, v);
            }
            *reinterpret_cast<u32x4_align2*>(dst + at) = w;
        } else {
            for (int e = 0; e < n / 2; ++e) {
                float u, v;
                round2(t[e], value(src[at + 2 * e], 0), value(src[at + 2 * e + 1], 0), u, v);
                dst[at + 2 * e] = to_bf16(u);
                dst[at + 2 * e + 1] = to_bf16(v);
            }
        }
    } else {
        const int half = a.rot / 2, at = 8 * c, n = min(8, half - at);
        const float2* t = turn + at;
        if (n == 8) {
            u32x4 x = *reinterpret_cast<const u32x4_align2*>(src + at), y = *reinterpret_cast<const u32x4_align2*>(src + half + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float u[2], v[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) round2(t[2 * e + i], value(x[e], i), value(y[e], i), u[i], v[i]);
                x[e] = pack_bf16x2(u[0], u[1]);
                y[e] = pack_bf16x2(v[0], v[1]);
            }
            *reinterpret_cast<u32x4_align2*>(dst + at) = x;
            *reinterpret_cast<u32x4_align2*>(dst + half + at) = y;
        } else {
            for (int e = 0; e < n; ++e) {
                float u, v;
                round2(t[e], value(src[at + e], 0), value(src[half + at + e], 0), u, v);
                dst[at + e] = to_bf16(u);
                dst[half + at + e] = to_bf16(v);
            }
        }
    }
}

// Row of the cache for a token, -1 if it has none.
__device__ __forceinline__ int64_t cache_row(const RopeArgs& a, int64_t token) {
    const int64_t p = a.positions[token], s = a.sequence != nullptr ? a.sequence[token] : token;
    if (s < 0 || s >= a.sequences || p < 0 || p >= (int64_t)a.width * a.page_size) return -1;
    const int at = (int)((uint32_t)p / (uint32_t)a.page_size), page = a.table[s * a.width + at];
    if (page < 0 || page >= a.pages) return -1;
    return (int64_t)page * a.page_size + (p - (int64_t)at * a.page_size);
}

template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a) {
    __shared__ float2 turn[kRopeTable];
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens_per_group;
    const int tokens = (int)min((int64_t)a.tokens_per_group, a.tokens - token0), half = a.rot / 2;
    for (int i = threadIdx.x; i < tokens * half; i += 256) {
        const int t = i / half;
        double turns = (double)a.positions[token0 + t] * a.freqs[i - t * half] * 0.15915494309189533577;
        turns -= rint(turns);
        float sn, cs;
        sincospif(2.f * (float)turns, &sn, &cs);
        turn[i] = float2{cs * a.amplitude, sn * a.amplitude * a.sign};
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * a.items; i += 256) {
        const int t = i / a.items;
        int c = i - t * a.items;
        const int64_t token = token0 + t;
        int w = 0;
        while (w < 2 && c >= a.s[w].heads * (a.s[w].turned + a.s[w].copied)) {
            c -= a.s[w].heads * (a.s[w].turned + a.s[w].copied);
            ++w;
        }
        const RopeStream& s = a.s[w];
        const int per = s.turned + s.copied, head = c / per;
        int64_t row = token;
        if (s.paged) {
            row = cache_row(a, token);
            if (row < 0) continue;
        }
        rope_piece<INTERLEAVED>(a, s, s.src + token * s.src_ts + head * s.src_hs, s.dst + row * s.dst_ts + head * s.dst_hs, c - head * per, turn + t * half);
    }
}

static int rope_launch(RopeArgs& a, int layout, void* stream) {
    a.items = 0;
    for (const RopeStream& s : a.s) a.items += s.heads * (s.turned + s.copied);
    if (a.items == 0) return QG_OK;       // in place, and nothing is turned
    // tokens of a workgroup: about two pieces per thread, if the launch keeps two workgroups per CU, and no more sines than fit
    int64_t per = 512 / a.items;
    if (per > a.tokens / 512) per = a.tokens / 512;
    if (a.rot > 0 && per > kRopeTable / (a.rot / 2)) per = kRopeTable / (a.rot / 2);
    a.tokens_per_group = (int)(per < 1 ? 1 : per);
    const dim3 grid((unsigned)((a.tokens + a.tokens_per_group - 1) / a.tokens_per_group));
    if (layout == QG_ROPE_INTERLEAVED) hipLaunchKernelGGL(k_rope<true>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(k_rope<false>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return check_launch();
}

static int check_rope(int64_t tokens, int d, int rot, int layout, float amplitude, const int64_t* positions, const double* freqs) {
    if (positions == nullptr || (rot != 0 && freqs == nullptr)) return QG_ERR_NULL;
    if (tokens <= 0 || tokens >= kAttnMaxTokens || d <= 0 || d > kRopeMaxD || rot < 0 || rot > d || rot % 2 != 0) return QG_ERR_SHAPE;
    if (layout != QG_ROPE_HALF && layout != QG_ROPE_INTERLEAVED) return QG_ERR_SHAPE;
    if (!(amplitude > -INFINITY && amplitude < INFINITY)) return QG_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(positions) & 7) || (reinterpret_cast<uintptr_t>(freqs) & 7)) return QG_ERR_ALIGN;
    return QG_OK;
}

// A stream that is turned (rot > 0) from one array to another.
static RopeStream rope_stream(const qg_heads* from, const qg_heads* to, int heads, int d, int rot, int layout) {
    RopeStream s = {};
    if (heads == 0) return s;
    s.src = from->data, s.src_ts = from->token_stride, s.src_hs = from->head_stride;
    s.dst = to->data, s.dst_ts = to->token_stride, s.dst_hs = to->head_stride;
    s.heads = heads;
    s.turned = layout == QG_ROPE_INTERLEAVED ? (rot + 7) / 8 : (rot / 2 + 7) / 8;
    const bool in_place = from->data == to->data && s.src_ts == s.dst_ts && s.src_hs == s.dst_hs;
    s.copied = in_place ? 0 : (d - rot + 7) / 8;
    return s;
}

static int rope(const qg_heads* q, int heads_q, const qg_heads* k, int heads_k, const int64_t* positions, const double* freqs, int64_t tokens,
                int d, int rot, int layout, float amplitude, const qg_heads* q_out, const qg_heads* k_out, float sign, void* stream) {
    if (heads_q <= 0 || heads_q > kAttnMaxHeads || heads_k < 0 || heads_k > kAttnMaxHeads || rot < 2) return QG_ERR_SHAPE;
    const int unit = d % 8 == 0 ? 8 : 1;       // (pieces of 16 bytes are read and written at any element)
    for (const qg_heads* x : {q, q_out})
        if (int e = check_heads(x, true, unit)) return e;
    for (const qg_heads* x : {k, k_out})
        if (int e = heads_k > 0 ? check_heads(x, true, unit) : QG_OK) return e;
    if (int e = check_rope(tokens, d, rot, layout, amplitude, positions, freqs)) return e;
    RopeArgs a = {};
    a.s[0] = rope_stream(q, q_out, heads_q, d, rot, layout);
    a.s[1] = rope_stream(k, k_out, heads_k, d, rot, layout);
    a.positions = positions, a.freqs = freqs, a.tokens = tokens, a.d = d, a.rot = rot, a.amplitude = amplitude, a.sign = sign;
    return rope_launch(a, layout, stream);
}

int check_cache(const qg_cache* c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->table == nullptr) return QG_ERR_NULL;
    if (c->pages <= 0 || c->page_size <= 0 || c->heads <= 0 || c->heads > kAttnMaxHeads || c->d <= 0 || c->d % 8 != 0 || c->d > kRopeMaxD) return QG_ERR_SHAPE;
    if (c->sequences <= 0 || c->sequences > kAttnMaxSequences || c->width <= 0) return QG_ERR_SHAPE;
    const int64_t most = int64_t(1) << 31;
    if (c->pages >= most || c->pages * c->page_size >= most || (int64_t)c->width * c->page_size >= most / 2 || (int64_t)c->sequences * c->width >= most)
        return QG_ERR_SHAPE;
    if (!aligned16(c->k) || !aligned16(c->v) || (reinterpret_cast<uintptr_t>(c->table) & 3)) return QG_ERR_ALIGN;
    return QG_OK;
}

}  // namespace qg

using namespace qg;

extern "C" int qg_rope_frequencies(int rot, double base, double factor, double context, double low, double high, double* out) {
    if (out == nullptr) return QG_ERR_NULL;
    if (rot < 2 || rot % 2 != 0 || rot > kRopeMaxD || !(base > 0) || !(factor > 0) || !(context >= 0)) return QG_ERR_SHAPE;
    if (context > 0 && !(low >= 0 && high > low)) return QG_ERR_SHAPE;
    for (int i = 0; i < rot / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot);
        double keep = 0;      // the share of the frequency as it is; the rest is divided
        if (context > 0) keep = std::fmin(1.0, std::fmax(0.0, (context * f / 6.28318530717958647692 - low) / (high - low)));
        out[i] = f * (keep + (1 - keep) / factor);
    }
    return QG_OK;
}

extern "C" int qg_rope_forward(const qg_heads* q, int heads_q, const qg_heads* k, int heads_k, const int64_t* positions, const double* freqs,
                               int64_t tokens, int d, int rot, int layout, float amplitude, const qg_heads* q_out, const qg_heads* k_out, void* stream) {
    return rope(q, heads_q, k, heads_k, positions, freqs, tokens, d, rot, layout, amplitude, q_out, k_out, 1.f, stream);
}

extern "C" int qg_rope_backward(const qg_heads* dq_out, int heads_q, const qg_heads* dk_out, int heads_k, const int64_t* positions, const double* freqs,
                                int64_t tokens, int d, int rot, int layout, float amplitude, const qg_heads* dq, const qg_heads* dk, void* stream) {
    return rope(dq_out, heads_q, dk_out, heads_k, positions, freqs, tokens, d, rot, layout, amplitude, dq, dk, -1.f, stream);
}

extern "C" int qg_cache_append(const qg_cache* c, const qg_heads* q, int heads_q, const qg_heads* k, const qg_heads* v, const int64_t* positions,
                               const int32_t* sequence, int64_t tokens, const double* freqs, int rot, int layout, float amplitude,
                               const qg_heads* q_out, void* stream) {
    if (int e = check_cache(c)) return e;
    if (heads_q < 0 || heads_q > kAttnMaxHeads) return QG_ERR_SHAPE;
    for (const qg_heads* x : {k, v})
        if (int e = check_heads(x, true)) return e;
    for (const qg_heads* x : {q, q_out})
        if (int e = heads_q > 0 ? check_heads(x, true) : QG_OK) return e;
    if (int e = check_rope(tokens, c->d, rot, layout, amplitude, positions, freqs)) return e;
    if (reinterpret_cast<uintptr_t>(sequence) & 3) return QG_ERR_ALIGN;
    RopeArgs a = {};
    a.s[0] = rope_stream(q, q_out, heads_q, c->d, rot, layout);
    const int64_t row = (int64_t)c->heads * c->d;
    const qg_heads to_k = {c->k, row, c->d}, to_v = {c->v, row, c->d};
    a.s[1] = rope_stream(k, &to_k, c->heads, c->d, rot, layout);
    a.s[2] = rope_stream(v, &to_v, c->heads, c->d, 0, layout);
    for (int w = 1; w < 3; ++w) a.s[w].paged = true;
    a.s[1].copied = (c->d - rot + 7) / 8, a.s[2].copied = c->d / 8;
    a.positions = positions, a.freqs = freqs, a.tokens = tokens, a.d = c->d, a.rot = rot, a.amplitude = amplitude, a.sign = 1.f;
    a.table = c->table, a.sequence = sequence, a.pages = c->pages, a.page_size = c->page_size, a.sequences = c->sequences, a.width = c->width;
    return rope_launch(a, layout, stream);
}
