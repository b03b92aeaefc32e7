"""CPU-only checks of the argument validation of the operators around the linear layer: every call below returns before its
first HIP call."""
import pytest

from paper_2407_08296_amd import qgalore as qg

FAKE = 0x10000          # non-null, 16-byte aligned, never dereferenced on the error paths


@pytest.fixture(scope="module")
def L():
    return qg.lib()


def caller(f, *args):
    """f with the given arguments, some of them replaced by position."""
    def call(**kw):
        a = list(args)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return f(*a)
    return call


def test_residual_norm_forward(L):
    # h, y, w_post, gate, kind, w_pre, scale, eps, tokens, d, ld, fp32, h_out, u, stream
    call = caller(L.qg_residual_norm_forward, FAKE, FAKE, FAKE, FAKE, 1, FAKE, 1.0, 1e-6, 16, 512, 512, 0, FAKE, FAKE, None)
    assert call(a0=None) == 1 and call(a5=None) == 1 and call(a12=None) == 1 and call(a3=None) == 1
    assert call(a1=None, a13=None) == 1                                   # nothing to compute
    assert call(a4=3) == 2 and call(a4=-1) == 2
    assert call(a8=0) == 2 and call(a8=1 << 22) == 2 and call(a9=0) == 2 and call(a9=16385) == 2
    assert call(a10=511) == 2 and call(a10=520) == 2 and call(a10=1 << 31) == 2   # below d; not a multiple of 16; too long
    for i in (0, 1, 2, 3, 5, 12, 13):
        assert call(**{f"a{i}": FAKE + 8}) == 4


def test_residual_norm_backward(L):
    # du, dh_next, h_next, y, w_post, gate, kind, w_pre, scale, eps, tokens, d, ld, fp32, dh, dy, dw_pre, dw_post, dgate, ws, bytes, stream
    nbytes = L.qg_residual_norm_workspace_bytes(16, 512)
    assert nbytes >= 2 * 512 * 4 and L.qg_residual_norm_workspace_bytes(0, 512) == 0 and L.qg_residual_norm_workspace_bytes(16, 16385) == 0
    assert L.qg_residual_norm_workspace_bytes(1 << 20, 512) <= 1 << 22     # does not grow with the tokens without end
    call = caller(L.qg_residual_norm_backward, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1, FAKE, 1.0, 1e-6, 16, 512, 512, 1, FAKE, FAKE, FAKE,
                  FAKE, FAKE, FAKE, nbytes, None)
    assert call(a0=None, a1=None) == 1 and call(a14=None) == 1 and call(a2=None) == 1 and call(a7=None) == 1 and call(a15=None) == 1
    assert call(a0=None) == 1                                             # dw_pre without du
    assert call(a4=None) == 1                                             # dw_post without w_post
    assert call(a5=None) == 1 and call(a6=0) == 1                         # gate missing; dgate without a gate
    assert call(a3=None) == 1                                             # dw_post and dgate without y
    assert call(a6=5) == 2 and call(a10=-1) == 2 and call(a11=0) == 2 and call(a12=8) == 2
    assert call(a19=None) == 5 and call(a20=nbytes - 1) == 5
    for i in (0, 1, 2, 3, 4, 5, 7, 14, 15, 16, 17, 18, 19):
        assert call(**{f"a{i}": FAKE + 4}) == 4
