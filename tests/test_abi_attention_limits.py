"""CPU-only checks of what the attention half refuses at the limits of its numbers."""
import pytest

from paper_2407_08296_amd import qgalore as qg
from test_abi_attention import ALIGN, FAKE, NULL, SHAPE, WORKSPACE, attention, cache, heads


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


def test_strides_of_rotary_heads_that_are_no_multiple_of_8(L):
    """Any strides and any element's address for such heads, as contiguous ones have; else multiples of 8.  (What is not refused for them is refused
    for its amplitude here.)"""
    for f in (L.qg_rope_forward, L.qg_rope_backward):
        def call(d, bad=None, at=0):
            x = [heads(FAKE, 3 * d, d)] * 4
            x[at] = x[at] if bad is None else bad
            return f(x[0], 3, x[1], 3, FAKE, FAKE, 10, d, 2, 0, float("nan"), x[2], x[3], None)
        for d in (2, 7, 20, 33, 100, 1023):
            assert call(d) == SHAPE
            for at in range(4):
                assert call(d, heads(FAKE + 2, 3 * d + 1, d + 1), at) == SHAPE and call(d, heads(FAKE + 1, 3 * d, d), at) == ALIGN
                assert call(d, heads(FAKE, 1 << 23, d), at) == SHAPE and call(d, heads(0), at) == NULL and call(d, heads(FAKE, -2, d), at) == SHAPE
        for d in (8, 64, 1024):
            for at in range(4):
                assert call(d, heads(FAKE + 2, 3 * d, d), at) == ALIGN and call(d, heads(FAKE, 3 * d + 1, d), at) == ALIGN and call(d, heads(FAKE, 3 * d, d + 4), at) == ALIGN
