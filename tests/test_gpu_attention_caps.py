"""Capped scores of every cap that is allowed, against the fp64 oracle.

Bounds.  Those of test_gpu_attention.py, but for the error of x = cap tanh(y), y = s / cap, s = scale q.k, which does not grow with the cap here:
  y is off by three roundings (the quotient scale / cap, a constant, the product), tanh by no more than that times |y|, so x by 3 2^-24 |s|;
  e = exp(-2 |y|) is off by one place, 2^-24 at most, and (1 - e) / (1 + e) by that; the cap multiplies it: cap 2^-24 up to a cap of 64, and from
    there on only where |y| >= 1/8, so 2^-24 / tanh(1/8) < 2^-20 of x;
  the sum, reciprocal, two products and log2(e): 8 2^-24 of x; the series up to 1/8 with its first term left out: 2^-22 and 4 roundings, less than that.
Together (cap <= 64: cap 2^-24) + (2^-20 + 2^-21) |s|, rounded up to 2^-19 |s|, on top of the product's (d + 16) 2^-24 scale |q|.|k|."""
import numpy as np
import pytest
import torch

from oracle import attention as A
from paper_2407_08296_amd import qgalore as qg
from test_gpu_attention import DEV, H, cu, np64, tensors

pytestmark = pytest.mark.gpu
CAPS = [2.0 ** -60, 1e-3, 30.0, 64.0, 64.00001, 200.0, 1e4, 1e6, 1e8, 1e10, 2.0 ** 60]


def error_of_scores(q, k, scale, cap):
    return (q.shape[-1] + 16) * 2.0 ** -24 * scale * (np.abs(q) @ np.abs(k).T) + (cap * 2.0 ** -24 if cap <= 64 else 0.0) + 2.0 ** -19 * scale * np.abs(q @ k.T)


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("slope", [0.0, 0.05])
def test_forward_and_backward(cap, d, slope):
    n = 330
    q, k, v, do = tensors(n, n, 2, 1, d, seed=d)
    slopes = torch.full((2,), slope, device=DEV) if slope else None
    o, lse = qg.attention_forward(q, k, v, cap=cap, slopes=slopes)
    grads = qg.attention_backward(do, q, k, v, o, lse, cap=cap, slopes=slopes)
    Q, K, V, G, O, L, dQ, dK, dV = (np64(t) for t in (q, k, v, do, o, lse, *grads))
    slope = float(np.float32(slope))
    scale, seen = d ** -0.5, A.visible(n, n)
    far = np.abs(np.arange(n)[:, None] - np.arange(n)[None])
    want_dk, want_dv, tol_dk, tol_dv = (np.zeros((n, d)) for _ in range(4))
    terms = 2 * n * 2.0 ** -24
    for h in range(2):
        qh, kh, vh, gh = Q[:, h], K[:, 0], V[:, 0], G[:, h]
        want, want_lse, p = A.attention(qh, kh, vh, scale, seen, cap, slope)
        e = np.where(seen, error_of_scores(qh, kh, scale, cap) + slope * far * 2.0 ** -23, 0.0).max(axis=1, keepdims=True)
        ep = e + (n + 16) * 2.0 ** -24 + np.abs(want_lse)[:, None] * 2.0 ** -22
        assert np.all(np.abs(L[h] - want_lse) <= ep[:, 0]), ("lse", float((np.abs(L[h] - want_lse) / ep[:, 0]).max()))
        tol = 1.01 * ((H + 2 * ep) * (p @ np.abs(vh)) + H * np.abs(want)) + 1e-30
        assert np.all(np.abs(O[:, h] - want) <= tol), ("o", float((np.abs(O[:, h] - want) / tol).max()))
        dq, dk, dv, ds = A.attention_gradients(gh, qh, kh, vh, scale, seen, cap, slope)
        inner = gh @ vh.T - (gh * want).sum(axis=1, keepdims=True)
        go = (np.abs(gh) * np.abs(want)).sum(axis=1, keepdims=True)
        eds = (H + 2 * ep) * np.abs(ds) + p * scale * ((d + n + 8) * 2.0 ** -24 * (np.abs(gh) @ np.abs(vh).T + go) + 2.0 ** -18 * np.abs(inner)) + np.abs(ds) * 2.0 ** -20
        tol = 1.01 * ((eds + n * 2.0 ** -24 * np.abs(ds)) @ np.abs(kh) + H * np.abs(dq) + H * go * (H + 2 * ep) * scale * (p @ np.abs(kh))) + 1e-30
        assert np.all(np.abs(dQ[:, h] - dq) <= tol), ("dq", float((np.abs(dQ[:, h] - dq) / tol).max()))
        want_dk += dk
        want_dv += dv
        tol_dk += (eds + terms * np.abs(ds)).T @ np.abs(qh)
        tol_dv += ((H + 2 * ep + terms) * p).T @ np.abs(gh)
    for name, got, want, tol in (("dk", dK[:, 0], want_dk, tol_dk), ("dv", dV[:, 0], want_dv, tol_dv)):
        tol = 1.01 * (tol + H * np.abs(want)) + 1e-30
        assert np.all(np.abs(got - want) <= tol), (name, float((np.abs(got - want) / tol).max()))


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("d", [64, 96, 128])
def test_paged(cap, d):
    n, page = 700, 16
    width = -(-n // page)
    q, k, v, _ = tensors(1, width * page, 4, 2, d, seed=d + 1)
    q = q.repeat(1, 2, 1)[:, :4].contiguous()
    table = torch.arange(width, dtype=torch.int32, device=DEV)[None]
    got = np64(qg.attention_paged(q, k.view(width, page, 2, d), v.view(width, page, 2, d), table, torch.tensor([n], dtype=torch.int32, device=DEV), cap=cap))[0]
    Q, K, V = np64(q)[0], np64(k)[:n], np64(v)[:n]
    for h in range(4):
        qh, kh, vh = Q[h:h + 1], K[:, h // 2], V[:, h // 2]
        want, want_lse, p = A.attention(qh, kh, vh, d ** -0.5, np.ones((1, n), bool), cap)
        ep = error_of_scores(qh, kh, d ** -0.5, cap).max() + (n + 16) * 2.0 ** -24 + abs(want_lse[0]) * 2.0 ** -22
        tol = 1.01 * ((H + 2 * ep) * (p @ np.abs(vh)) + H * np.abs(want)) + 1e-30
        assert np.all(np.abs(got[h] - want[0]) <= tol[0]), float((np.abs(got[h] - want[0]) / tol[0]).max())


def test_zero_scores_under_the_smallest_cap_and_values_that_are_not_finite():
    """A score of 0 stays 0 whatever the cap; a NaN is not taken for a score."""
    q, k, v, do = tensors(70, 70, 1, 1, 64, 3)
    for cap in (2.0 ** -60, 2.0 ** 60):
        o, lse = qg.attention_forward(torch.zeros_like(q), k, v, cap=cap)
        assert torch.equal(lse[0], qg.attention_forward(torch.zeros_like(q), k, v)[1][0]) and bool(torch.isfinite(o).all())
        assert all(bool(torch.isfinite(g).all()) for g in qg.attention_backward(do, torch.zeros_like(q), k, v, o, lse, cap=cap))
    for cap in (30.0, 1e6):
        bad = k.clone()
        bad[40] = float("nan")
        o, lse = qg.attention_forward(q, bad, v, cap=cap)
        assert bool(torch.isnan(lse[0, 40:]).all()) and bool(torch.isnan(o[40:]).all())


def test_refused_caps():
    q, k, v, do = tensors(40, 40, 2, 1, 64, 4)
    o, lse = qg.attention_forward(q, k, v)
    pages = k.view(4, 10, 1, 64)
    table, n = torch.arange(4, dtype=torch.int32, device=DEV)[None], torch.tensor([40], dtype=torch.int32, device=DEV)
    for cap in (2.0 ** -61, 1e-45, 2.0 ** 61, 3e38):
        for call in (lambda: qg.attention_forward(q, k, v, cap=cap), lambda: qg.attention_backward(do, q, k, v, o, lse, cap=cap),
                     lambda: qg.attention_paged(q[:1], pages, pages, table, n, cap=cap)):
            with pytest.raises(qg.QGError):
                call()
