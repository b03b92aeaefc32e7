"""The fp64 attention oracle against its definitions written out, and its gradients against central differences."""
import math

import numpy as np
import pytest

from oracle import attention as A

KINDS = [dict(), dict(cap=2.0), dict(slope=0.3), dict(cap=1.5, slope=-0.2)]


def data(n_q, n_k, d, seed=0):
    rng = np.random.default_rng(seed)
    return rng.normal(size=(n_q, d)), rng.normal(size=(n_k, d)), rng.normal(size=(n_k, d))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_k,mask", [(5, 5, dict()), (3, 7, dict(window=2)), (6, 4, dict()), (5, 5, dict(prefix=3)), (4, 6, dict(causal=False))])
def test_rows_written_out(kind, n_q, n_k, mask):
    q, k, v = data(n_q, n_k, 4)
    seen = A.visible(n_q, n_k, **mask)
    o, lse, _ = A.attention(q, k, v, 0.5, seen, **kind)
    for i in range(n_q):
        p, terms = i + n_k - n_q, {}
        for j in range(n_k):
            s = 0.5 * sum(q[i][e] * k[j][e] for e in range(4))
            if kind.get("cap"):
                s = kind["cap"] * math.tanh(s / kind["cap"])
            hidden = mask.get("causal", True) and j > p and j >= mask.get("prefix", 0)
            if not hidden and not (mask.get("window") and p - j >= mask["window"]):
                terms[j] = math.exp(s - kind.get("slope", 0.0) * abs(p - j))
        if not terms:
            assert lse[i] == -math.inf and not o[i].any()
            continue
        total = sum(terms.values())
        assert abs(lse[i] - math.log(total)) < 1e-12
        for e in range(4):
            assert abs(o[i][e] - sum(t * v[j][e] for j, t in terms.items()) / total) < 1e-12


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_q,n_k,mask", [(4, 4, dict()), (5, 3, dict()), (3, 5, dict(window=2)), (4, 4, dict(prefix=2)), (3, 4, dict(causal=False))])
def test_gradients_are_differences(kind, n_q, n_k, mask):
    q, k, v = data(n_q, n_k, 3, 1)
    do = np.random.default_rng(2).normal(size=(n_q, 3))
    seen = A.visible(n_q, n_k, **mask)
    f = lambda *x: float((A.attention(*x, 0.7, seen, **kind)[0] * do).sum())
    got = A.attention_gradients(do, q, k, v, 0.7, seen, **kind)[:3]
    h = 1e-5
    for w, g in enumerate(got):
        for at in np.ndindex(g.shape):
            x = [a.copy() for a in (q, k, v)]
            x[w][at] += h
            up = f(*x)
            x[w][at] -= 2 * h
            assert abs((up - f(*x)) / (2 * h) - g[at]) < 1e-7      # third derivatives times h^2, and 1e-16 / h


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_turns_pairs(layout):
    """Complex multiplication; lengths kept; the backward pass undoes it; scores depend on the distance alone."""
    rng = np.random.default_rng(3)
    x, freqs = rng.normal(size=(3, 2, 8)), A.rope_frequencies(6)
    pos = np.array([0, 5, 1000000])
    y = A.rope(x, pos, freqs, layout, 2.0)
    for t in range(3):
        for i, f in enumerate(freqs):
            a, b = (i, i + 3) if layout == "half" else (2 * i, 2 * i + 1)
            z = 2.0 * (x[t, :, a] + 1j * x[t, :, b]) * np.exp(1j * pos[t] * f)
            assert np.abs(y[t, :, a] - z.real).max() < 1e-9 and np.abs(y[t, :, b] - z.imag).max() < 1e-9
    assert np.array_equal(y[..., 6:], x[..., 6:]) and np.array_equal(A.rope(x, [0] * 3, freqs, layout), x)
    assert np.abs(A.rope(A.rope(x, pos, freqs, layout), pos, freqs, layout, backward=True) - x).max() < 1e-9
    q, k = rng.normal(size=(2, 1, 1, 8))
    dots = [float((A.rope(q, [p + 7], freqs, layout) * A.rope(k, [p], freqs, layout)).sum()) for p in (0, 10, 500)]
    assert max(dots) - min(dots) < 1e-9


def test_frequencies():
    f = A.rope_frequencies(8)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001])
    assert np.allclose(A.rope_frequencies(8, factor=4.0), f / 4)
    g = A.rope_frequencies(8, factor=4.0, context=2 * np.pi * 250, low=1.0, high=4.0)      # turns: 250, 25, 2.5, 0.25
    assert np.allclose(g, [1.0, 0.1, 0.01 * (0.5 + 0.5 / 4), 0.001 / 4])


def test_places_of_a_cache():
    table = [[3, 0, -1], [9, 2, 1]]
    assert A.cache_place(table, 0, 5, 4, 5) == (0, 1) and A.cache_place(table, 0, 8, 4, 5) is None and A.cache_place(table, 0, 12, 4, 5) is None
    assert A.cache_place(table, 1, 0, 4, 5) is None and A.cache_place(table, 2, 0, 4, 5) is None and A.cache_place(table, 1, -1, 4, 5) is None
    rows, end = A.paged_rows(table, 1, 7, 4, 5, window=4)
    assert rows == [(4, (2, 0)), (5, (2, 1)), (6, (2, 2))] and end == 7
