"""CPU-only checks of what the attention half refuses at the limits of its numbers."""
import pytest

from paper_2407_08296_amd import qgalore as qg
from test_abi_attention import FAKE, SHAPE, WORKSPACE, attention, cache, heads


@pytest.fixture(scope="module")
def L():
    return qg.lib()


def test_scales_and_caps(L):
    """A scale, and a cap that is not 0, from 2^-60 to 2^60: their quotient is a number of fp32.  (A call that is not refused for them is refused for
    its workspace here.)"""
    h = heads()

    def codes(**kw):
        a, c = attention(**kw), cache()
        scale, cap = kw.get("scale", 0.125), kw.get("cap", 0.0)
        return {L.qg_attention_backward(a, h, h, h, h, h, FAKE, h, h, h, None, 0, None), L.qg_attention_paged(c, FAKE, h, 8, scale, cap, 0, None, h, None, 0, None)}
    for cap in (2.0 ** -61, 1e-45, 2.0 ** 61, 3e38):
        assert codes(cap=cap) == {SHAPE}, cap
        assert L.qg_attention_forward(attention(cap=cap), h, h, h, h, FAKE, None, 0, None) == SHAPE
    for scale in (2.0 ** -61, 1e-45, 2.0 ** 61, 3e38):
        assert codes(scale=scale) == {SHAPE} and codes(scale=scale, cap=5.0) == {SHAPE}, scale
    for cap in (0.0, 2.0 ** -60, 2.0 ** 60):
        for scale in (2.0 ** -60, 1.0, 2.0 ** 60):
            assert codes(cap=cap, scale=scale) == {WORKSPACE}, (cap, scale)
