"""Which outputs of the attention half's binding share memory with an input, another output or themselves: against sets of addresses, on the CPU."""
import random

import pytest
import torch

from paper_2407_08296_amd import qgalore as qg


def elements(t):
    """Addresses, in elements, of a [tokens][heads][d] view."""
    at = t.data_ptr() // 2
    T, H, d = t.shape
    ts, hs, _ = t.stride()
    return [at + i * ts + h * hs + e for i in range(T) for h in range(H) for e in range(d)]


def some_view(rng, base, d, ts=None):
    T, H = rng.choice([1, 1, 2, 3, 7]), rng.choice([1, 2, 3, 5])
    ts = rng.choice([0, d, 2 * d, 3 * d + 8, 96, 120]) if ts is None else ts
    hs = rng.choice([0, 8, d, d + 8, 2 * d, 48])
    room = base.numel() - ((T - 1) * ts + (H - 1) * hs + d)
    return base.as_strided((T, H, d), (ts, hs, 1), 8 * rng.randrange(max(1, room // 8)))


def test_overlap_of_any_two_views():
    rng = random.Random(1)
    base = torch.empty(2000, dtype=torch.bfloat16)
    seen = [0, 0, 0]
    for _ in range(6000):
        d = rng.choice([8, 16, 24])
        x = some_view(rng, base, d)
        y = some_view(rng, base, d, ts=x.stride(0) if rng.random() < 0.8 else None)
        want = not set(elements(x)).isdisjoint(elements(y))
        got = qg._overlap(qg._span(x), qg._span(y))
        assert got == qg._overlap(qg._span(y), qg._span(x))
        alike = x.stride(0) == y.stride(0) or x.shape[0] == 1 or y.shape[0] == 1
        assert got == want if alike else got or not want, (x.shape, x.stride(), y.shape, y.stride(), x.storage_offset(), y.storage_offset())
        seen[2 if not alike else int(want)] += 1
    assert min(seen) > 200


def test_outputs_that_overlap_themselves():
    rng = random.Random(2)
    base = torch.empty(2000, dtype=torch.bfloat16)
    seen = [0, 0]
    for _ in range(3000):
        t = some_view(rng, base, rng.choice([8, 16]))
        at = elements(t)
        want = len(set(at)) < len(at)
        if want:
            with pytest.raises(qg.QGError):
                qg._written(t, t, "out")
        else:
            assert qg._written(t, t, "out") is t
        seen[want] += 1
    assert min(seen) > 200


def test_slices_of_one_layers_output_lie_apart():
    x = torch.empty(50, 8 * 64, dtype=torch.bfloat16)
    q, k, v = x[:, :256].view(50, 4, 64), x[:, 256:384].view(50, 2, 64), x[:, 384:].view(50, 2, 64)
    qg._apart((q, k, v), ())
    qg._apart((q, k), (v, None))
    qg._apart((q, k), (q, k), (q, k))                             # in place
    qg._apart((q.view(50, 4, 64),), (q, k, v), (q,))              # the same place by another view
    qg._apart((q[::2],), (k, k[::2], v[1::3]))                    # other columns of some of the rows
    outside = torch.empty(4, 100, 64, dtype=torch.bfloat16).transpose(0, 1)
    qg._apart((outside[:40], outside[40:]), ())                   # heads outside the tokens
    for outs, ins, places in [((q, k), (q, k), ()), ((k, q), (q[:, :2], k), (q[:, :2], k)), ((q, q), (), ()), ((q[1:],), (q[:-1],), (q[:-1],)), ((q[:, 1:],), (q[:, :3],), (q[:, :3],)),
                              ((outside[:41], outside[40:]), (), ())]:
        with pytest.raises(qg.QGError):
            qg._apart(outs, ins, places)
