"""Attention and the paged cache at sizes where 32-bit offsets, or the rules for how many workgroups there are, would go wrong."""
import pytest
import torch

from paper_2407_08296_amd import qgalore as qg
from test_gpu_attention import DEV, check, cu, tensors
from test_gpu_rope_cache import check_paged, normal

pytestmark = pytest.mark.gpu


def far_apart(t, big, at, token_stride, head_stride):
    """t's values at these strides from element `at` of big on."""
    x = big.as_strided(t.shape, (token_stride, head_stride, 1), at)
    x.copy_(t)
    return x


@pytest.mark.parametrize("token_stride,head_stride", [((1 << 23) - 8, 256), (256, 1 << 31)])
def test_arrays_past_32_bits(token_stride, head_stride):
    """The longest rows that are allowed, 300 of them (2^31.2 elements), and heads 2^31 elements apart: the bits of contiguous tensors, forward and backward.
    Every array of the call lies in one buffer, side by side."""
    T, heads, heads_k, d = 300, 3, 1, 64
    q, k, v, do = tensors(T, T, heads, heads_k, d, 1)
    bounds = cu([170, 130])
    o, lse = qg.attention_forward(q, k, v, bounds)
    grads = qg.attention_backward(do, q, k, v, o, lse, bounds)
    side = heads * head_stride if head_stride < token_stride else T * token_stride      # elements of an array before the next may begin
    span = (T - 1) * token_stride + (heads - 1) * head_stride + 8 * side + d
    big = torch.empty(span, dtype=torch.bfloat16, device=DEV)
    assert span > 1 << 31
    at = iter(range(0, 8 * side, side))
    bq, bk, bv, bdo = (far_apart(t, big, next(at), token_stride, head_stride) for t in (q, k, v, do))
    places = [big.as_strided(t.shape, (token_stride, head_stride, 1), next(at)) for t in (q, *grads)]
    o2, lse2 = qg.attention_forward(bq, bk, bv, bounds, out=places[0])
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    got = qg.attention_backward(bdo, bq, bk, bv, o2, lse2, bounds, out=tuple(places[1:]))
    assert all(torch.equal(a, b) for a, b in zip(got, grads))
    check(q, k, v, do, [170, 130], o=o, lse=lse, grads=grads)


def test_a_long_batch_past_32_bits():
    """2^31 elements of contiguous q: its last sequence against the oracle, the others zeros."""
    T, heads, d = 530000, 32, 128
    lengths = [52947] * 10 + [530]
    q = torch.zeros(T, heads, d, dtype=torch.bfloat16, device=DEV)
    assert q.numel() > 1 << 31 and sum(lengths) == T
    k, v, do = (torch.zeros_like(q) for _ in range(3))
    last = tensors(530, 530, heads, heads, d, 2)
    for t, x in zip((q, k, v, do), last):
        t[-530:] = x
    bounds = cu(lengths)
    o, lse = qg.attention_forward(q, k, v, bounds, window=64)
    grads = qg.attention_backward(do, q, k, v, o, lse, bounds, window=64)
    check(*last, [530], o=o[-530:], lse=lse[:, -530:], grads=[t[-530:] for t in grads], window=64)
    assert not o[:-530].any() and not any(t[:-530].any() for t in grads)


@pytest.mark.parametrize("window", [0, 1500])
def test_paged_one_workgroup_for_all_parts(window):
    """More than 4096 sequences and key heads: one workgroup walks all parts of its sequence and writes o by itself."""
    sequences, page = 4200, 16
    lengths = [2500 if i in (0, 17, 4199) else i % 50 for i in range(sequences)]
    pages = sum(-(-n // page) for n in lengths)
    kp, vp = normal(pages, page, 1, 64, seed=1, std=1.5), normal(pages, page, 1, 64, seed=2)
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(3)).tolist()
    table, at = torch.full((sequences, 160), -1, dtype=torch.int32), 0
    for i, n in enumerate(lengths):
        for j in range(-(-n // page)):
            table[i, j], at = ids[at], at + 1
    q = normal(sequences, 2, 64, seed=4, std=1.5)
    got = qg.attention_paged(q, kp, vp, table.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), window=window)
    check_paged(q, kp, vp, table, lengths, got, window=window)
