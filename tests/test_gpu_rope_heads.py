"""Rotary positions of heads whose size is no multiple of 8, as contiguous tensors have them and as slices; bounds of test_gpu_rope_cache.py."""
import pytest
import torch

from paper_2407_08296_amd import qgalore as qg
from test_gpu_rope_cache import DEV, normal, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,heads_k,d,rot", [(5, 3, 1, 2, 2), (40, 2, 2, 7, 6), (17, 3, 1, 20, 20), (700, 4, 2, 33, 32), (9, 5, 5, 100, 50), (3, 2, 1, 1023, 1022), (1, 1, 0, 36, 2)])
def test_rope(tokens, heads, heads_k, d, rot, layout):
    guard = torch.full((3, tokens, heads, d), 3.0, dtype=torch.bfloat16, device=DEV)
    q, k = normal(tokens, heads, d, seed=1), normal(tokens, heads_k, d, seed=2) if heads_k else None
    pos, freqs = torch.arange(tokens, device=DEV) * 977, qg.rope_frequencies(rot)
    for f, backward in ((qg.rope_forward, False), (qg.rope_backward, True)):
        a, b = f(q, k, pos, freqs, layout, 0.75)
        turned(q, a, pos, freqs, layout, 0.75, backward)
        if k is not None:
            turned(k, b, pos, freqs, layout, 0.75, backward)
        f(q, None, pos, freqs, layout, 0.75, out=(guard[1], None))
        assert torch.equal(guard[1], a) and bool((guard[0] == 3).all()) and bool((guard[2] == 3).all())
        x = q.clone()
        f(x, None, pos, freqs, layout, 0.75, out=(x, None))
        assert torch.equal(x, a)
        wide = torch.full((tokens, heads, d + 3), 5.0, dtype=torch.bfloat16, device=DEV)      # a slice from the second element on: every address is unaligned
        wide[:, :, 1:d + 1] = q
        x = wide[:, :, 1:d + 1]
        assert torch.equal(f(x, None, pos, freqs, layout, 0.75)[0], a)
        f(x, None, pos, freqs, layout, 0.75, out=(x, None))
        assert torch.equal(x, a) and bool((wide[:, :, 0] == 5).all()) and bool((wide[:, :, d + 1:] == 5).all())
