"""Outputs of the attention half that share memory with something else: refused where workgroups would read what others write, right where they may."""
import pytest
import torch

from paper_2407_08296_amd import qgalore as qg
from test_gpu_attention import DEV, tensors
from test_gpu_rope_cache import check_paged, make_cache, normal

pytestmark = pytest.mark.gpu


def test_refusals():
    T, heads, heads_k, d = 60, 4, 2, 64
    q, k, v, do = tensors(T, T, heads, heads_k, d, 1)
    k4, v4 = (t.repeat(1, 2, 1) for t in (k, v))
    o, lse = qg.attention_forward(q, k4, v4)
    pos, freqs = torch.arange(T, device=DEV), qg.rope_frequencies(d)
    kp, vp, table = make_cache(12, 16, heads_k, d, 4, 3)
    n = torch.full((3,), 40, dtype=torch.int32, device=DEV)
    big = torch.zeros(2 * T, heads, d, dtype=torch.bfloat16, device=DEV)
    new = lambda: torch.empty_like(q)
    grads = lambda *out: (lambda: qg.attention_backward(do, q, k4, v4, o, lse, out=out))
    bad = [lambda: qg.attention_forward(q, k4, v4, out=q), lambda: qg.attention_forward(q, k4, v4, out=k4), lambda: qg.attention_forward(q, k4, v4, out=v4),
           lambda: qg.attention_forward(big[:T], k4, v4, out=big[T - 1:2 * T - 1]),
           grads(q, new(), new()), grads(new(), k4, new()), grads(new(), new(), v4), grads(do, new(), new()), grads(o, new(), new()), grads(k4, new(), new()),
           grads(*[new()] * 2, new()), grads(big[:T], big[T:], big[1:T + 1]),
           lambda: qg.rope_forward(q, k4, pos, freqs, out=(k4, q)), lambda: qg.rope_forward(q, k4, pos, freqs, out=(q, q)), lambda: qg.rope_forward(q, q, pos, freqs, out=(q, q)),
           lambda: qg.rope_forward(big[:T], None, pos, freqs, out=(big[1:T + 1], None)), lambda: qg.rope_backward(q, k4, pos, freqs, out=(k4, new())),
           lambda: qg.rope_forward(q, None, pos, freqs, out=(big.as_strided((T, heads, d), (heads * d, 32, 1)), None)),
           lambda: qg.cache_append(q[:3], k[:3], v[:3], pos[:3], kp, kp, table), lambda: qg.cache_append(q[:3, :2], k[:3], v[:3], pos[:3], kp, vp, table, out=k[:3]),
           lambda: qg.cache_append(q[:3, :2], k[:3], v[:3], pos[:3], kp, vp, table, out=vp[0, :3]),
           lambda: qg.attention_paged(q[:3, :2], kp, vp, table, n, out=kp[1, :3]), lambda: qg.attention_paged(big[:3], kp, vp, table, n, out=big[1:4])]
    before = [t.clone() for t in (q, k4, v4, do, o, big, k, kp, vp)]
    for i, call in enumerate(bad):
        with pytest.raises(qg.QGError, match="overlap"):
            call()
            pytest.fail(f"call {i}")
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (q, k4, v4, do, o, big, k, kp, vp)))


@pytest.mark.parametrize("lengths", [[40, 7, 0], [3000, 700, 1]])
def test_paged_in_place(lengths):
    """o over q, with one share of a sequence and with several."""
    width = 190
    kp, vp, table = make_cache(3 * width, 16, 2, 64, width, 3)
    q = normal(3, 8, 64, seed=5, std=1.5)
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    want = qg.attention_paged(q, kp, vp, table, n)
    x = q.clone()
    assert qg.attention_paged(x, kp, vp, table, n, out=x) is x and torch.equal(x, want)
    x = q.clone()
    qg.attention_paged(x, kp, vp, table, n, out=x.view(3, 8, 64))
    assert torch.equal(x, want)
    check_paged(q, kp, vp, table, lengths, want)


def test_rows_of_the_pages_appended_elsewhere():
    """A page's rows as the tokens of other sequences (none of the places written is read)."""
    kp, vp, table = make_cache(20, 16, 2, 64, 4, 3)
    spare = next(p for p in range(20) if p not in table.flatten().tolist())
    want_k, want_v = kp.clone(), vp.clone()
    for t in range(3):
        want_k[table[t, 1], 4], want_v[table[t, 1], 4] = kp[spare, t], vp[spare, t]
    qg.cache_append(None, kp[spare, :3], vp[spare, :3], torch.full((3,), 20, device=DEV), kp, vp, table)
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
