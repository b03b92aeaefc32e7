"""Boundaries of packed sequences that descend: nothing is written but the rows of the sequences that they name, and nothing outside the arrays."""
import pytest
import torch

from paper_2407_08296_amd import qgalore as qg
from test_gpu_attention import DEV, tensors

pytestmark = pytest.mark.gpu
T, HEADS, HEADS_K, D = 300, 2, 1, 64


def guarded(heads):
    """[3][tokens][heads][d] of a value; the middle is an output, the rest stays."""
    return torch.full((3, T, heads, D), 3.0, dtype=torch.bfloat16, device=DEV)


def both(inputs, bounds):
    """o, lse, dq, dk, dv, each between guards."""
    q, k, v, do = inputs
    outs = [guarded(h) for h in (HEADS, HEADS, HEADS_K, HEADS_K)]
    lse = torch.full((3, HEADS, T), 3.0, device=DEV)
    a = qg._attention(q, k, v, bounds, None, True, None, 0.0, None, 0, None)
    heads = lambda t: qg._heads(t)
    ws = torch.empty(max(qg.lib().qg_attention_forward_workspace_bytes(a), 16), dtype=torch.uint8, device=DEV)
    qg._check(qg.lib().qg_attention_forward(a, heads(q), heads(k), heads(v), heads(outs[0][1]), lse[1].data_ptr(), ws.data_ptr(), ws.numel(), qg._stream()))
    qg.attention_backward(do, q, k, v, outs[0][1], lse[1], bounds, out=tuple(t[1] for t in outs[1:]))
    torch.cuda.synchronize()
    for t in (*outs, lse):
        assert bool((t[0] == 3).all()) and bool((t[2] == 3).all())
    return (*(t[1] for t in outs), lse[1])


@pytest.mark.parametrize("b", [[0, 300, 0, 300, 0], [0, 200, 100, 300], [5, -7, 2 ** 31 - 1, 50], [300, 0, 300, 0], [-1, -1, -1, -1], [0, 300, 0, 300, 0, 300, 0],
                               [0, 299, 1, 298, 2, 297, 3]])
def test_nothing_outside_the_arrays(b):
    both(tensors(T, T, HEADS, HEADS_K, D, 19), torch.tensor(b, dtype=torch.int32, device=DEV))


def test_a_sequence_that_ends_ahead_of_its_start_has_no_rows():
    """[0, 300), [300, 0), [0, 300): the second is empty, and the others are one and the same, twice.  (Its tile ahead of row 300 was taken for rows without
    keys: zeros over the others' rows, or theirs over it, whichever came last.)"""
    inputs = tensors(T, T, HEADS, HEADS_K, D, 20)
    want = both(inputs, torch.tensor([0, 300, 300, 300], dtype=torch.int32, device=DEV))
    got = both(inputs, torch.tensor([0, 300, 0, 300], dtype=torch.int32, device=DEV))
    assert all(torch.equal(x, y) for x, y in zip(got, want))
