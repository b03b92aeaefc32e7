"""Attention over packed sequences, forward and backward, against the fp64 oracle, each output element against a bound of its own.

Bounds.  h = 2^-8 is half a step of bf16.  A score's error: the product of d terms in fp32 and the steps after it, e = (d + 16) 2^-24
scale |q|.|k| (+ cap 2^-21: tanh by an exponential and a reciprocal of one step each, + slope distance 2^-23); probabilities are then off by the
factor e + (keys + 16) 2^-24 (the sum; exponentials; lse's own rounding, |lse| 2^-23).  p is rounded to bf16 for the product with v:
    |o - want|  <= (h + 2 e') sum p |v| + h |o|                                   (o's own rounding)
    |lse - want| <= e + (keys + 16) 2^-24 + |lse| 2^-22
    |dv - want| <= (h + 2 e') sum p |do| + h |dv|
ds = p (do.v - delta) factor scale, rounded to bf16.  delta is formed from o as stored and corrected by the sum of the row's p (do.v - delta), fp32:
    |ds - want| <= (h + 2 e') |ds| + p scale ((d + keys + 8) 2^-24 (|do|.|v| + |do|.|o|) + 2^-19 |do.v - delta| if capped)
    |dq - want| <= sum |ds's error| |k| + h |dq| + (h |do|.|o|) (h + 2 e') scale sum p |k|         (the correction and its bf16 p), dk without that;
fp32 sums over n terms add n 2^-24 of the sum of magnitudes.
(All first order; 1 % on top for the products of errors.)"""
import math

import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2407_08296_amd import qgalore as qg

pytestmark = pytest.mark.gpu
DEV = "cuda"
H = 2.0 ** -8
np64 = lambda t: t.detach().float().cpu().numpy().astype(np.float64)


def tensors(tokens, tokens_k, heads, heads_k, d, seed, std=1.5):
    gen = torch.Generator().manual_seed(seed)
    r = lambda n, h, s: (torch.randn(n, h, d, generator=gen) * s).bfloat16().to(DEV)
    return r(tokens, heads, std), r(tokens_k, heads_k, std), r(tokens_k, heads_k, 1.0), r(tokens, heads, 0.1)


def cu(lengths):
    return torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int32, device=DEV)


def check(q, k, v, do, lengths, lengths_k=None, causal=True, scale=None, cap=0.0, slopes=None, window=0, prefix=None, o=None, lse=None, grads=None):
    """Every element of o, lse and, if given, grads against the bounds above; rows behind the last sequence: zeros."""
    Q, K, V, G = (np64(t) for t in (q, k, v, do))
    heads, heads_k, d = Q.shape[1], K.shape[1], Q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    O, L = np64(o), np64(lse)
    want_dk, want_dv, tol_dk, tol_dv = (np.zeros_like(K) for _ in range(4))
    if grads is not None:
        dQ, dK, dV = (np64(t) for t in grads)
    q0 = k0 = 0
    for s, n in enumerate(lengths):
        m = n if lengths_k is None else lengths_k[s]
        seen = A.visible(n, m, causal, window, 0 if prefix is None else min(max(int(prefix[s]), 0), m)) if n * m else np.zeros((n, m), bool)
        far = np.abs(np.arange(n)[:, None] + m - n - np.arange(m)[None])
        for h in range(heads):
            g = h // (heads // heads_k)
            qh, kh, vh, gh = Q[q0:q0 + n, h], K[k0:k0 + m, g], V[k0:k0 + m, g], G[q0:q0 + n, h]
            slope = 0.0 if slopes is None else float(slopes[h])
            want, want_lse, p = A.attention(qh, kh, vh, scale, seen, cap, slope)
            e = (d + 16) * 2.0 ** -24 * scale * (np.abs(qh) @ np.abs(kh).T) + cap * 2.0 ** -21 + abs(slope) * far * 2.0 ** -23
            e = np.where(seen, e, 0.0).max(axis=1, initial=0.0, keepdims=True)
            top = np.where(np.isfinite(want_lse), np.abs(want_lse), 0.0)[:, None]
            ep = e + (m + 16) * 2.0 ** -24 + top * 2.0 ** -22
            got, got_lse = O[q0:q0 + n, h], L[h, q0:q0 + n]
            tol = 1.01 * ((H + 2 * ep) * (p @ np.abs(vh)) + H * np.abs(want)) + 1e-30
            assert np.all(np.abs(got - want) <= tol), ("o", s, h, float((np.abs(got - want) / tol).max()))
            empty = ~seen.any(axis=1)
            assert np.all(got[empty] == 0) and np.all(got_lse[empty] == -np.inf)
            off = np.abs(got_lse[~empty] - want_lse[~empty])
            assert np.all(off <= ep[~empty, 0]), ("lse", s, h, float(off.max()))
            if grads is None:
                continue
            dq, dk, dv, ds = A.attention_gradients(gh, qh, kh, vh, scale, seen, cap, slope)
            inner = gh @ vh.T - (gh * want).sum(axis=1, keepdims=True)
            go = (np.abs(gh) * np.abs(want)).sum(axis=1, keepdims=True)
            eds = (H + 2 * ep) * np.abs(ds) + p * scale * ((d + m + 8) * 2.0 ** -24 * (np.abs(gh) @ np.abs(vh).T + go)
                                                         + (2.0 ** -19 * np.abs(inner) if cap else 0.0)) + np.abs(ds) * 2.0 ** -20
            tol = 1.01 * ((eds + m * 2.0 ** -24 * np.abs(ds)) @ np.abs(kh) + H * np.abs(dq) + H * go * (H + 2 * ep) * scale * (p @ np.abs(kh))) + 1e-30
            off = np.abs(dQ[q0:q0 + n, h] - dq)
            assert np.all(off <= tol), ("dq", s, h, float((off / tol).max()))
            want_dk[k0:k0 + m, g] += dk
            want_dv[k0:k0 + m, g] += dv
            terms = n * heads // heads_k * 2.0 ** -24
            tol_dk[k0:k0 + m, g] += (eds + terms * np.abs(ds)).T @ np.abs(qh)
            tol_dv[k0:k0 + m, g] += ((H + 2 * ep + terms) * p).T @ np.abs(gh)
        q0, k0 = q0 + n, k0 + m
    assert not O[q0:].any() and np.all(L[:, q0:] == -np.inf)
    if grads is not None:
        for name, got, want, tol in (("dk", dK, want_dk, tol_dk), ("dv", dV, want_dv, tol_dv)):
            tol = 1.01 * (tol + H * np.abs(want)) + 1e-30
            assert np.all(np.abs(got - want) <= tol), (name, float((np.abs(got - want) / tol).max()))
        assert not dQ[q0:].any() and not dK[k0:].any() and not dV[k0:].any()


def run(lengths, heads=2, heads_k=2, d=64, seed=0, lengths_k=None, pad=0, pad_k=None, backward=True, **how):
    T, Tk = sum(lengths) + pad, sum(lengths if lengths_k is None else lengths_k) + (pad if pad_k is None else pad_k)
    q, k, v, do = tensors(T, Tk, heads, heads_k, d, seed)
    bounds = None if len(lengths) == 1 and not pad and lengths_k is None else cu(lengths)
    bounds_k = None if lengths_k is None else cu(lengths_k)
    o, lse = qg.attention_forward(q, k, v, bounds, bounds_k, **how)
    grads = qg.attention_backward(do, q, k, v, o, lse, bounds, bounds_k, **how) if backward else None
    torch.cuda.synchronize()
    check(q, k, v, do, lengths, lengths_k, o=o, lse=lse, grads=grads, **how)


def slopes_of(heads):
    return torch.tensor([0.5 ** h for h in range(heads)], device=DEV)


# (tokens, tokens_k, heads, heads_k, d, sequences, flags: 1 causal, 2 cap, 4 slopes): calls that the host cuts into parts, and every kernel
PARTS = [(2048, 2048, 2, 1, 128, 1, 1), (16, 3000, 2, 2, 64, 1, 1), (1, 3000, 1, 1, 80, 1, 1), (700, 700, 3, 1, 96, 1, 0), (3000, 40, 2, 1, 64, 1, 0), (1500, 1500, 1, 1, 72, 1, 7),
         (1200, 1200, 6, 1, 128, 1, 3), (2100, 2100, 8, 8, 64, 1, 1)]
KERNELS = [(150, 150, 2, 1, d, 1, f) for d in (64, 96, 128) for f in (1, 3, 5, 7)]


@pytest.mark.parametrize("tokens,tokens_k,heads,heads_k,d,sequences,flags", PARTS + KERNELS)
def test_every_kernel(tokens, tokens_k, heads, heads_k, d, sequences, flags):
    run([tokens], heads=heads, heads_k=heads_k, d=d, lengths_k=None if tokens == tokens_k else [tokens_k], causal=bool(flags & 1), cap=6.0 if flags & 2 else 0.0,
        slopes=slopes_of(heads) if flags & 4 else None, seed=tokens)


@pytest.mark.parametrize("how", [dict(), dict(window=300), dict(prefix=True, cap=9.0)])
def test_parts_of_packed_sequences(how):
    """Parts where sequences are of very different lengths: some have steps for every part, some for none; a padded end."""
    how = dict(how, prefix=torch.tensor([900, 0, 3, 40], dtype=torch.int32, device=DEV)) if how.get("prefix") else how
    run([1900, 0, 5, 700], heads=2, heads_k=1, d=64, pad=50, seed=21, **how)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 600])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths(n, causal):
    run([n], causal=causal, seed=n)


@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 104, 120, 128])
def test_head_sizes(d):
    run([150], heads=2, heads_k=1, d=d, seed=d)


@pytest.mark.parametrize("heads,heads_k", [(1, 1), (3, 3), (8, 2), (5, 1), (12, 4)])
def test_grouped_heads(heads, heads_k):
    run([70, 90], heads=heads, heads_k=heads_k, d=64, seed=heads)


HOW = [dict(cap=5.0), dict(cap=200.0), dict(slopes=True), dict(cap=8.0, slopes=True), dict(window=1), dict(window=37), dict(window=64, cap=5.0), dict(window=10 ** 9),
       dict(window=90, slopes=True), dict(causal=False, slopes=True), dict(causal=False, cap=5.0), dict(prefix=(0, 0, 0, 0)), dict(prefix=(1, 0, 100, 40)),
       dict(prefix=(999, -3, 65, 130), slopes=True), dict(scale=0.01), dict(scale=1.0)]


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("how", range(len(HOW)))
def test_scores_and_masks(how, d):
    how = dict(HOW[how])
    if how.get("slopes"):
        how["slopes"] = slopes_of(2) * (1 if d != 80 else -0.01)      # (one that favours far keys, too)
    if "prefix" in how:
        how["prefix"] = torch.tensor(how["prefix"], dtype=torch.int32, device=DEV)
    run([1, 64, 100, 170], heads=2, heads_k=1, d=d, pad=9, seed=3, **how)


@pytest.mark.parametrize("lengths", [[0], [0, 0, 5], [3, 0, 0, 130, 0], [1] * 70, [128, 128], [127, 129, 1], [64] * 5])
@pytest.mark.parametrize("pad", [0, 1, 300])
def test_packed_lengths(lengths, pad):
    if sum(lengths) + pad == 0:
        pad = 3
    run(lengths, heads=2, heads_k=1, d=64, pad=pad, seed=len(lengths))


@pytest.mark.parametrize("n", [300, 5000])
def test_many_sequences(n):
    """More boundaries than one look takes, of lengths 0 to 3."""
    lengths = [int(v) for v in np.random.default_rng(n).integers(0, 4, n)]
    run(lengths, heads=1, heads_k=1, d=64, pad=2, seed=n)


@pytest.mark.parametrize("lengths,lengths_k", [([5], [200]), ([130], [400]), ([200], [50]), ([64, 1, 0, 40], [64, 300, 20, 0]), ([33, 100], [129, 70])])
@pytest.mark.parametrize("how", [dict(), dict(causal=False), dict(window=40), dict(slopes=True, cap=6.0), dict(prefix=30)])
def test_other_keys_than_queries(lengths, lengths_k, how):
    """A chunk of queries behind keys that are there already; more queries than keys (the first see none); none of one or the other."""
    how = dict(how, slopes=slopes_of(4)) if how.get("slopes") else how
    how = dict(how, prefix=torch.full((len(lengths),), how["prefix"], dtype=torch.int32, device=DEV)) if how.get("prefix") else how
    run(lengths, heads=4, heads_k=2, d=64, lengths_k=lengths_k, pad=4, pad_k=11, seed=7, **how)


def test_one_sequence_of_other_keys_without_boundaries():
    q, k, v, do = tensors(40, 90, 2, 1, 64, 5)
    o, lse = qg.attention_forward(q, k, v)
    check(q, k, v, do, [40], [90], o=o, lse=lse, grads=qg.attention_backward(do, q, k, v, o, lse))


def test_long_sequence():
    """Far from the diagonal: 63 whole steps ahead of the masked one, maxima raised along the way."""
    q, k, v, do = tensors(4100, 4100, 1, 1, 64, 11)
    ramp = torch.linspace(0.2, 4.0, 4100, device=DEV)[:, None, None]
    k = (k * ramp).bfloat16()
    o, lse = qg.attention_forward(q, k, v)
    check(q, k, v, do, [4100], o=o, lse=lse, grads=qg.attention_backward(do, q, k, v, o, lse))


def test_scores_far_below_and_above_zero():
    """Rows whose scores are all very negative, or very large: the running maximum carries them."""
    q, k, v, do = tensors(200, 200, 2, 2, 64, 12, std=0.3)
    shift = torch.ones(64, device=DEV) * 5
    for sign in (-1, 1):
        ks = (k + sign * shift).bfloat16()
        qs = (q + shift).bfloat16()
        o, lse = qg.attention_forward(qs, ks, v, scale=1.0)
        check(qs, ks, v, do, [200], scale=1.0, o=o, lse=lse, grads=qg.attention_backward(do, qs, ks, v, o, lse, scale=1.0))


def test_strides_and_outputs_given():
    """q, k and v as slices of one layer's output, heads outside the tokens, outputs into slices; what lies between stays."""
    T, heads, heads_k, d = 140, 4, 2, 64
    q, k, v, do = tensors(T, T, heads, heads_k, d, 13)
    o0, lse0 = qg.attention_forward(q, k, v)
    g0 = qg.attention_backward(do, q, k, v, o0, lse0)
    qkv = torch.cat([t.reshape(T, -1) for t in (q, k, v)], 1)
    split = lambda x: (x[:, :heads * d].view(T, heads, d), x[:, heads * d:(heads + heads_k) * d].view(T, heads_k, d),
                       x[:, (heads + heads_k) * d:].view(T, heads_k, d))
    sq, sk, sv = split(qkv)
    wide = torch.full((T, heads, 2 * d), 7.0, dtype=torch.bfloat16, device=DEV)
    o1, lse1 = qg.attention_forward(sq, sk, sv, out=wide[:, :, :d])
    dqkv = torch.full_like(qkv, 7.0)
    qg.attention_backward(do, sq, sk, sv, o1, lse1, out=split(dqkv))
    assert torch.equal(o1, o0) and torch.equal(lse1, lse0) and bool((wide[:, :, d:] == 7).all())
    assert all(torch.equal(a, b) for a, b in zip(split(dqkv), g0))
    outside = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    o2, lse2 = qg.attention_forward(*(outside(t) for t in (q, k, v)), out=outside(torch.empty_like(q)))
    g2 = qg.attention_backward(outside(do), *(outside(t) for t in (q, k, v)), o2, lse2, out=tuple(outside(torch.empty_like(t)) for t in (q, k, v)))
    assert torch.equal(o2, o0) and torch.equal(lse2, lse0) and all(torch.equal(a, b) for a, b in zip(g2, g0))
    shared = k[:, :1].expand(T, 2, d)                   # one key head for all, expanded: an input may be
    o3, _ = qg.attention_forward(q, shared, v)
    o4, _ = qg.attention_forward(q, shared.contiguous(), v)
    assert torch.equal(o3, o4)


def test_what_lies_outside_the_sequences_is_not_read():
    q, k, v, do = tensors(300, 300, 2, 2, 128, 14)
    for t in (q, k, v, do):
        t[250:] = float("nan")
    bounds = cu([100, 150])
    o, lse = qg.attention_forward(q, k, v, bounds)
    grads = qg.attention_backward(do, q, k, v, o, lse, bounds)
    assert all(bool(torch.isfinite(t).all()) for t in (o, *grads)) and bool((o[250:] == 0).all()) and bool((grads[1][250:] == 0).all())
    # one sequence's values never reach another's
    k[:100] = float("inf")
    v[:100] = float("nan")
    o2, lse2 = qg.attention_forward(q, k, v, bounds)
    assert torch.equal(o2[100:], o[100:]) and torch.equal(lse2[:, 100:], lse[:, 100:])


def test_the_same_bits_again_and_on_another_stream():
    q, k, v, do = tensors(1000, 1000, 8, 2, 128, 15)
    bounds = cu([300, 77, 623])

    def once():
        o, lse = qg.attention_forward(q, k, v, bounds)
        return (o, lse, *qg.attention_backward(do, q, k, v, o, lse, bounds))
    first = once()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        again = once()
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_captured_and_replayed_with_other_boundaries():
    """The launch goes by the tokens and the number of sequences; lengths may change between replays."""
    q, k, v, do = tensors(500, 500, 4, 2, 64, 16)
    bounds = cu([100, 400])
    ws = torch.empty(16 * 500 * 4 * 130 * 4, dtype=torch.uint8, device=DEV)

    def both():
        o, lse = qg.attention_forward(q, k, v, bounds, workspace=ws)
        return (o, lse, *qg.attention_backward(do, q, k, v, o, lse, bounds, workspace=ws))
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for lengths in ([100, 400], [250, 250], [7, 300], [0, 500]):
        bounds.copy_(cu(lengths))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, both()))
        torch.cuda.synchronize()
        check(q, k, v, do, lengths, o=got[0], lse=got[1], grads=got[2:])


def test_a_training_pass_against_automatic_differentiation():
    """The whole formula's gradients: a rounding of an operand and one of the result, each h / sqrt(3) of the size in the mean."""
    T, d = 130, 64
    q, k, v, do = tensors(T, T, 1, 1, d, 17)
    leaves = [t[:, 0].double().requires_grad_() for t in (q, k, v)]
    x = leaves[0] @ leaves[1].t().contiguous() * d ** -0.5
    x = x.masked_fill(torch.ones(T, T, device=DEV).triu(1).bool(), -math.inf)
    p = torch.softmax(x, 1)
    (p @ leaves[2]).backward(do[:, 0].double())
    o, lse = qg.attention_forward(q, k, v)
    got = qg.attention_backward(do, q, k, v, o, lse)
    for g, leaf in zip(got, leaves):
        assert float((g[:, 0].double() - leaf.grad).norm()) <= 0.9 * H * float(leaf.grad.norm())


def test_boundaries_that_make_no_sense():
    """Descending, negative, past the end: what comes out is of no use, but nothing outside the arrays is touched."""
    q, k, v, do = tensors(300, 300, 2, 1, 64, 19)
    guard = torch.full((3, 300, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    for b in ([0, 200, 100, 300], [5, -7, 2 ** 31 - 1, 50], [300, 0, 300, 0], [-1, -1, -1, -1]):
        bounds = torch.tensor(b, dtype=torch.int32, device=DEV)
        out = guard[1]
        o, lse = qg.attention_forward(q, k, v, bounds, out=out)
        qg.attention_backward(do, q, k, v, o, lse, bounds)
        torch.cuda.synchronize()
        assert bool((guard[0] == 3).all()) and bool((guard[2] == 3).all())


def test_refusals():
    q, k, v, do = tensors(40, 40, 4, 2, 64, 18)
    o, lse = qg.attention_forward(q, k, v)
    bad = [lambda: qg.attention_forward(q, k, v[:, :1]), lambda: qg.attention_forward(q[:, :3], k, v), lambda: qg.attention_forward(q.float(), k, v),
           lambda: qg.attention_forward(q.cpu(), k, v), lambda: qg.attention_forward(q, k, v, cu([40]).long()),
           lambda: qg.attention_forward(q, k, v, window=-1), lambda: qg.attention_forward(q, k, v, causal=False, window=5),
           lambda: qg.attention_forward(q, k, v, cap=-1.0), lambda: qg.attention_forward(q, k, v, scale=0.0), lambda: qg.attention_forward(q, k, v, scale=math.nan),
           lambda: qg.attention_forward(q, k, v, slopes=torch.ones(3, device=DEV)), lambda: qg.attention_forward(q, k, v, prefix=cu([1])[:1], window=3),
           lambda: qg.attention_forward(q, k[:30], v[:30], cu([40])), lambda: qg.attention_forward(q, k, v, None, cu([40])),
           lambda: qg.attention_forward(q[:, :, :60], k[:, :, :60], v[:, :, :60]), lambda: qg.attention_forward(q[:, :, 1:33], k[:, :, :32], v[:, :, :32]),
           lambda: qg.attention_forward(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2)),
           lambda: qg.attention_forward(q, k, v, out=o[:1].expand(40, 4, 64)), lambda: qg.attention_forward(q, k, v, workspace=torch.empty(0, dtype=torch.uint8, device=DEV)) and
           qg.attention_backward(do, q, k, v, o, lse, workspace=torch.empty(8, dtype=torch.uint8, device=DEV)),
           lambda: qg.attention_backward(do[:30], q, k, v, o, lse), lambda: qg.attention_backward(do, q, k, v, o, lse[:, :30])]
    for call in bad:
        with pytest.raises((qg.QGError, ValueError)):
            call()
