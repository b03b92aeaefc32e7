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


def test_int8_linear_act(L):
    # x, Wq, Ws, bias, residual, act, tokens, m, n, ld_n, ld_m, group, z, y, stream
    call = caller(L.qg_int8_linear_act_forward, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 16, 512, 256, 0, 0, 256, FAKE, FAKE, None)
    for i in (0, 1, 2, 13):
        assert call(**{f"a{i}": None}) == 1
    assert call(a5=4) == 2 and call(a5=-1) == 2
    assert call(a6=0) == 2 and call(a7=-1) == 2 and call(a8=0) == 2 and call(a6=1 << 20, a7=1 << 12) == 2
    assert call(a9=255) == 2 and call(a9=264) == 2 and call(a10=520) == 2
    assert call(a11=128) == 3
    for i in (0, 1, 2, 3, 4, 12, 13):
        assert call(**{f"a{i}": FAKE + 2}) == 4
    nbytes = L.qg_int8_linear_act_workspace_bytes(16, 512, 256)
    assert nbytes >= 512 * 4 and L.qg_int8_linear_act_workspace_bytes(0, 512, 256) == 0 and L.qg_int8_linear_act_workspace_bytes(1 << 20, 1 << 20, 8) == 0
    # dy, z, x, Wq, Ws, act, tokens, m, n, ld_n, ld_m, group, dx, G, dbias, ws, bytes, stream
    call = caller(L.qg_int8_linear_act_backward, FAKE, FAKE, FAKE, FAKE, FAKE, 3, 16, 512, 256, 0, 0, 256, FAKE, FAKE, FAKE, FAKE, nbytes, None)
    for i in (0, 1, 2, 3, 4):
        assert call(**{f"a{i}": None}) == 1
    assert call(a12=None, a13=None, a14=None) == 1
    assert call(a5=9) == 2 and call(a6=0) == 2 and call(a9=8) == 2 and call(a10=500) == 2 and call(a11=64) == 3
    assert call(a15=None) == 5 and call(a16=nbytes - 1) == 5
    for i in (0, 1, 2, 3, 4, 12, 13, 14, 15):
        assert call(**{f"a{i}": FAKE + 8}) == 4


def test_int8_gated(L):
    # x, Wgq, Wgs, Wuq, Wus, act, tokens, m, n, ld_n, ld_m, group, zg, zu, y, stream
    call = caller(L.qg_int8_gated_forward, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 16, 512, 256, 0, 0, 256, FAKE, FAKE, FAKE, None)
    for i in (0, 1, 2, 3, 4, 12, 13, 14):
        assert call(**{f"a{i}": None}) == 1          # zg without zu, and the other way round, too
    assert call(a5=4) == 2 and call(a6=0) == 2 and call(a9=250) == 2 and call(a10=513) == 2 and call(a11=32) == 3
    for i in (0, 1, 2, 3, 4, 12, 13, 14):
        assert call(**{f"a{i}": FAKE + 4}) == 4
    # dy, zg, zu, x, Wgq, Wgs, Wuq, Wus, act, tokens, m, n, ld_n, ld_m, group, dx, Gg, Gu, ws, bytes, stream
    nbytes = L.qg_int8_gated_workspace_bytes(16, 512, 256)
    assert nbytes >= 2 * 16 * 512 * 2 and L.qg_int8_gated_workspace_bytes(0, 512, 256) == 0
    call = caller(L.qg_int8_gated_backward, *[FAKE] * 8, 2, 16, 512, 256, 0, 0, 256, FAKE, FAKE, FAKE, FAKE, nbytes, None)
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 16, 17):
        assert call(**{f"a{i}": None}) == 1
    assert call(a15=None, a16=None, a17=None) == 1
    assert call(a8=7) == 2 and call(a10=0) == 2 and call(a12=1) == 2 and call(a13=528 + 1) == 2 and call(a14=1) == 3
    assert call(a18=None) == 5 and call(a19=nbytes - 1) == 5
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 15, 16, 17, 18):
        assert call(**{f"a{i}": FAKE + 8}) == 4


def test_head_loss(L):
    nbytes = L.qg_head_loss_workspace_bytes(16, 64, 1000)
    assert nbytes >= 16 * 64 * 2 + 16 * 1000 * 2
    for bad in ((0, 64, 1000), (16, 0, 1000), (16, 64, -1), (1 << 24, 64, 1000), (16, 65536, 1000), (16, 64, 1 << 24), (1 << 20, 64, 1 << 18),
                (1 << 23, 2048, 1000), (16, 8192, 1 << 24), (16, 65535, 1 << 22)):
        assert L.qg_head_loss_workspace_bytes(*bad) == 0
    # a long batch over a wide vocabulary: far below its logits in 16 bits
    assert L.qg_head_loss_workspace_bytes(65536, 4096, 128000) < 65536 * 128000 * 2 // 8
    # x, W, labels, tokens, h, vocab, ld, loss, lse, ws, bytes, stream
    call = caller(L.qg_head_loss_forward, FAKE, FAKE, FAKE, 16, 64, 1000, 0, FAKE, FAKE, FAKE, nbytes, None)
    for i in (0, 1, 2, 7, 8):
        assert call(**{f"a{i}": None}) == 1
    assert call(a3=0) == 2 and call(a4=0) == 2 and call(a5=0) == 2 and call(a6=63) == 2 and call(a6=72) == 2
    for i in (0, 1, 9):
        assert call(**{f"a{i}": FAKE + 8}) == 4
    assert call(a2=FAKE + 4) == 4 and call(a7=FAKE + 2) == 4 and call(a8=FAKE + 1) == 4
    assert call(a2=FAKE + 8, a7=FAKE + 4, a8=FAKE + 4, a10=64) == 5      # labels by 8, numbers by 4: on to the next check
    assert call(a9=None) == 5 and call(a10=64) == 5
    # x, W, labels, lse, dloss, tokens, h, vocab, ld, dx, dW, ws, bytes, stream
    call = caller(L.qg_head_loss_backward, FAKE, FAKE, FAKE, FAKE, FAKE, 16, 64, 1000, 0, FAKE, FAKE, FAKE, nbytes, None)
    for i in (0, 1, 2, 3, 4):
        assert call(**{f"a{i}": None}) == 1
    assert call(a9=None, a10=None) == 1
    assert call(a5=-4) == 2 and call(a8=65) == 2
    for i in (0, 1, 2, 9, 10, 11):
        assert call(**{f"a{i}": FAKE + 4}) == 4
    assert call(a3=FAKE + 2) == 4 and call(a4=FAKE + 2) == 4
    assert call(a2=FAKE + 8, a3=FAKE + 4, a4=FAKE + 12, a12=64) == 5
    assert call(a11=None) == 5 and call(a12=64) == 5
