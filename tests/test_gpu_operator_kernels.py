"""The operators around the linear layer at sizes where the host takes each of their kernels (tests/test_launch_kernels.py holds these lists
against the kernels that the library has): whole and ragged tiles of every size, weight gradients by direct loads, the head's tokens put
together.  Workspaces are filled with NaN first, so that a number read that nothing wrote shows.

Bars: those of test_gpu_linear_act.py, whose checks run here on other sizes, and of test_gpu_head_loss.py, here against a reference in fp64
on the GPU."""
import numpy as np
import pytest
import torch

import test_gpu_linear_act as layer
from oracle import layers as O
from paper_2407_08296_amd import qgalore as qg

pytestmark = pytest.mark.gpu
DEV = "cuda"
U24 = 2.0 ** -24

# (tokens, m, n) of the activated layer: the contraction over eight waves and over four; 64 x 64 in one group and in two; 128 x 64 in two; 128 x
# 128 in two, in one with one register set and with two; whole and ragged
ACT_FORWARD = [(64, 1024, 256), (256, 2048, 128), (512, 2048, 256), (512, 2048, 512), (1024, 2048, 640), (1000, 2040, 960), (1024, 4096, 768),
               (1000, 4090, 770), (512, 8320, 64), (512, 16640, 64), (500, 16600, 72)]
# ... of its weight gradient by direct loads: whole columns, rows of x that start aligned and that are copied, one token
ACT_DIRECT = [(70, 5461, 2048), (65, 5463, 2051), (1, 8192, 1024), (96, 4096, 2048)]
# ... of the pair
GATED_FORWARD = [(64, 1024, 256), (512, 2048, 1024), (500, 4090, 800)]
# its dx in 128 x 128 tiles, whole and in parts of the contraction, and in 256 x 256, whole and ragged
GATED_DX = [(512, 128, 256), (256, 1024, 256), (4096, 64, 4096), (4090, 100, 4096)]
GATED_DIRECT = [(100, 5461, 1024), (33, 5461, 1027), (1, 5504, 1024), (64, 4096, 1024), (300, 2736, 1501)]

# (tokens, h, vocab) of the head: 128 x 128 and 256 x 256 tiles of whole sizes, dx in 256 x 256, more than 64 tokens per workgroup that puts
# them together
HEAD = [(512, 64, 8192), (1024, 64, 16384), (4096, 4096, 256), (4100, 4100, 300), (70000, 16, 300), (130, 40, 530000)]
# ... whose forward pass puts the tokens that have a loss together
TOGETHER = [(1000, 1100, 32003), (300, 4100, 30001), (2100, 1030, 16001), (1024, 1088, 32000), (512, 2112, 32000), (70000, 61, 8100), (65, 16400, 32500)]


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("tokens,m,n", ACT_FORWARD)
def test_act_forward(tokens, m, n, act):
    layer.test_act_forward(tokens, m, n, act)


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("tokens,m,n", GATED_FORWARD)
def test_gated_forward(tokens, m, n, act):
    layer.test_gated_forward(tokens, m, n, act)


@pytest.mark.parametrize("tokens,m,n", GATED_DX + GATED_DIRECT)
def test_gated_backward(tokens, m, n):
    layer.test_gated_backward(tokens, m, n, "silu")


@pytest.mark.parametrize("tokens,m,n", ACT_DIRECT)
def test_act_backward(tokens, m, n):
    layer.test_act_backward(tokens, m, n, "gelu")


def nan_bytes(count):
    return torch.full((count,), 255, dtype=torch.uint8, device=DEV)      # bf16 and fp32 NaN


def padded(t, ld):
    p = torch.full((t.shape[0], ld), 77 if t.dtype is torch.int8 else float("nan"), dtype=t.dtype, device=DEV)
    p[:, :t.shape[1]] = t
    return p


@pytest.mark.parametrize("tokens,m,n,ld_n", [(33, 5461, 1027, 0), (33, 5461, 1027, 1040), (100, 5461, 1024, 0), (64, 4096, 1024, 1040), (1, 8192, 1024, 0),
                                             (150, 2050, 1200, 0)])
def test_backward_in_a_workspace_of_nan(tokens, m, n, ld_n):
    """Both layers' backward passes, x, W, dx and G dense and at a pitch (odd rows then need no copy); padding holds NaN and keeps it."""
    g = torch.Generator().manual_seed(tokens + m + n)
    (wg, Wg), (wu, Wu) = layer.weight(g, m, n), layer.weight(g, m, n)
    x, dy, zg, zu = layer.normal(g, tokens, n), layer.normal(g, tokens, m, std=0.05), layer.normal(g, tokens, m, std=2.0), layer.normal(g, tokens, m)
    ld = ld_n or n
    xp, gp, up = padded(x, ld), padded(wg[0], ld), padded(wu[0], ld)
    dx, dx2, G, Gg, Gu = (torch.full((rows, ld), 7.0, dtype=torch.bfloat16, device=DEV) for rows in (tokens, tokens, m, m, m))
    db = torch.full((m,), 7.0, device=DEV)
    L, at, st = qg.lib(), (lambda t: t.data_ptr()), torch.cuda.current_stream().cuda_stream
    wa, wp = (nan_bytes(f(tokens, m, n)) for f in (L.qg_int8_linear_act_workspace_bytes, L.qg_int8_gated_workspace_bytes))
    assert L.qg_int8_linear_act_backward(at(dy), at(zg), at(xp), at(gp), at(wg[1]), 3, tokens, m, n, ld_n, 0, 256, at(dx), at(G), at(db), at(wa),
                                         wa.numel(), st) == 0
    assert L.qg_int8_gated_backward(at(dy), at(zg), at(zu), at(xp), at(gp), at(wg[1]), at(up), at(wu[1]), 2, tokens, m, n, ld_n, 0, 256, at(dx2), at(Gg),
                                    at(Gu), at(wp), wp.numel(), st) == 0
    X, DY, ZG, ZU = (layer.f64(t) for t in (x, dy, zg, zu))
    r, rss = 4 * 2.0 ** -8, layer.rss
    dz = DY * O.act(ZG, "gelu")[1]
    layer.check(dx[:, :n], dz @ Wg, (r + 4 * m * U24) * rss(dz, Wg) + 1e-6 * rss(DY, Wg))
    layer.check(G[:, :n], dz.T @ X, (r + 4 * tokens * U24) * rss(dz.T, X) + 1e-6 * rss(DY.T, X))
    assert np.all(np.abs(layer.f64(db) - dz.sum(0)) <= 8 * (1 + np.sqrt(tokens)) * U24 * np.abs(dz).sum(0) + 5e-7 * np.abs(DY).sum(0))
    a, da = O.act(ZG, "silu")
    dzg, dzu = DY * ZU * da, DY * a
    layer.check(dx2[:, :n], dzg @ Wg + dzu @ Wu, (r + 4 * m * U24) * (rss(dzg, Wg) + rss(dzu, Wu)) + 1e-6 * (rss(DY * ZU, Wg) + rss(DY * ZG, Wu)))
    layer.check(Gg[:, :n], dzg.T @ X, (r + 4 * tokens * U24) * rss(dzg.T, X) + 1e-6 * rss((DY * ZU).T, X))
    layer.check(Gu[:, :n], dzu.T @ X, (r + 4 * tokens * U24) * rss(dzu.T, X) + 1e-6 * rss((DY * ZG).T, X))
    for t in (dx, dx2, G, Gg, Gu):
        assert bool((t[:, n:] == 7).all())


# ---------------------------------------------------------------- head
def head_inputs(tokens, h, vocab, ignored, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + tokens + h + vocab)
    x = torch.randn(tokens, h, device=DEV, generator=g).bfloat16()
    W = (torch.randn(vocab, h, device=DEV, generator=g) * (2 / h ** 0.5)).bfloat16()
    labels = torch.randint(0, vocab, (tokens,), device=DEV, generator=g)
    labels[torch.rand(tokens, device=DEV, generator=g) < ignored] = -100
    if ignored < 1:
        labels[0], labels[1], labels[2], labels[3], labels[tokens - 1] = 0, vocab - 1, vocab, 1 << 40, vocab // 2
    on = (labels >= 0) & (labels < vocab)
    x = torch.where(on[:, None], x, torch.full_like(x, float("nan")))         # (what has no loss may hold anything)
    return x, W, labels, on, torch.where(on, torch.randn(tokens, device=DEV, generator=g), float("nan"))


def head_reference(x, W, labels, on):
    """fp64, of the tokens that have a loss: x, W, logits, lse, loss, and the noise of a logit (see test_gpu_head_loss.py)."""
    X, V = x[on].double(), W.double()
    z = X @ V.t().contiguous()
    lse = torch.logsumexp(z, 1)
    loss = lse - z.gather(1, labels[on][:, None])[:, 0]
    noise = 4 * X.shape[1] * U24 * float(((X * X).sum(1).max() * (V * V).sum(1).max()).sqrt()) if len(X) else 0.0
    return X, V, z, lse, loss, noise


def workspace(tokens, h, vocab):
    return nan_bytes(qg.lib().qg_head_loss_workspace_bytes(tokens, h, vocab))


@pytest.mark.parametrize("ignored", [0.0, 0.5, 0.97, 1.0])
@pytest.mark.parametrize("tokens,h,vocab", TOGETHER + HEAD)
def test_head_forward(tokens, h, vocab, ignored):
    x, W, labels, on, _ = head_inputs(tokens, h, vocab, ignored)
    loss, lse = qg.head_loss_forward(x, W, labels, workspace=workspace(tokens, h, vocab))
    assert not loss[~on].any() and not lse[~on].any()
    _, _, _, want, wloss, noise = head_reference(x, W, labels, on)
    bar = noise + (np.log2(vocab) + 40) * U24 * (1 + want.abs())
    assert bool(((lse[on].double() - want).abs() <= bar).all())
    assert bool(((loss[on].double() - wloss).abs() <= 2 * bar + 4 * U24 * wloss.abs()).all())
    again = qg.head_loss_forward(x, W, labels)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)


@pytest.mark.parametrize("ignored", [0.0, 0.5, 0.97])
@pytest.mark.parametrize("tokens,h,vocab", [(1000, 1100, 32003), (1024, 1088, 32000), (65, 16400, 32500)] + HEAD)
def test_head_backward(tokens, h, vocab, ignored):
    x, W, labels, on, dloss = head_inputs(tokens, h, vocab, ignored, seed=1)
    lse = qg.head_loss_forward(x, W, labels)[1]
    dx, dW = qg.head_loss_backward(x, W, labels, lse, dloss, workspace=workspace(tokens, h, vocab))
    assert not dx[~on].any()
    X, V, z, want_lse, _, noise = head_reference(x, W, labels, on)
    g = dloss[on].double()[:, None]
    p = (z - want_lse[:, None]).exp_()
    del z
    rel = 2 * noise + 2 * (np.log2(vocab) + 40) * U24 * (1 + want_lse.abs())[:, None]
    perr = g.abs() * p * rel
    p.scatter_add_(1, labels[on][:, None], torch.full((len(X), 1), -1.0, dtype=torch.float64, device=DEV))
    dl = p * g
    for got, a, e, b in ((dx[on], dl, perr, V), (dW, dl.t().contiguous(), perr.t().contiguous(), X)):
        want = a @ b
        bar = 2.0 ** -8 * want.abs() + (4 * 2.0 ** -8 + 4 * a.shape[1] ** 0.5 * U24) * ((a * a) @ (b * b)).sqrt() + e @ b.abs()
        assert bool(((got.double() - want).abs() <= bar).all())
    again = qg.head_loss_backward(x, W, labels, lse, dloss)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dW)


@pytest.mark.parametrize("tokens,h,vocab", [(300, 4100, 30001), (1000, 1100, 32003), (512, 64, 8192)])
def test_head_without_any_token(tokens, h, vocab):
    x, W, labels, on, dloss = head_inputs(tokens, h, vocab, 1.0)
    assert not on.any()
    dx, dW = qg.head_loss_backward(x, W, labels, torch.zeros(tokens, device=DEV), dloss, workspace=workspace(tokens, h, vocab))
    assert not dx.any() and not dW.any()


def test_tokens_put_together_in_a_graph():
    """The forward pass that puts tokens together, captured and replayed with other labels than it was captured with."""
    tokens, h, vocab = 1000, 1100, 32003
    x, W, labels, on, dloss = head_inputs(tokens, h, vocab, 0.0)
    x, dloss = torch.nan_to_num(x), torch.nan_to_num(dloss)
    ws = workspace(tokens, h, vocab)

    def both():
        loss, lse = qg.head_loss_forward(x, W, labels, workspace=ws)
        return (loss, lse) + qg.head_loss_backward(x, W, labels, lse, dloss, workspace=ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for every in (1, 3, 400):
        labels.copy_(torch.where(torch.arange(tokens, device=DEV) % every == 0, torch.arange(tokens, device=DEV) * 31, -1))
        want = [t.clone() for t in both()]
        for t in got:
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_long_batch_whose_dz_passes_2_to_the_31_elements():
    """Rows of dz are 64 elements apart in the workspace whatever m is: 40000003 tokens reach past 2^31 of them.  dy is zero but for some
    hundred rows at both ends and around 2^31 / 64, so that G has few terms and dx few rows."""
    tokens, m, n = 40000003, 5, 8
    gen = torch.Generator().manual_seed(16)
    (wg, Wg), (wu, Wu) = layer.weight(gen, m, n), layer.weight(gen, m, n)
    g = torch.Generator(device=DEV).manual_seed(17)
    x, zg, zu = (torch.randn(tokens, k, device=DEV, generator=g, dtype=torch.bfloat16) for k in (n, m, m))
    at = torch.cat([torch.arange(v, v + 200, device=DEV) for v in (0, (1 << 25) - 100, tokens - 200)])
    dy = torch.zeros(tokens, m, dtype=torch.bfloat16, device=DEV)
    dy[at] = torch.randn(len(at), m, device=DEV, generator=g).bfloat16()
    X, DY, ZG, ZU = (layer.f64(t[at]) for t in (x, dy, zg, zu))
    r, rss, k = 4 * 2.0 ** -8, layer.rss, len(at)
    dz = DY * O.act(ZG, "silu")[1]
    dx, G, db = qg.int8_linear_act_backward(dy, zg, x, *wg, act="silu", want_dbias=True)
    layer.check(dx[at], dz @ Wg, (r + 4 * m * U24) * rss(dz, Wg) + 1e-6 * rss(DY, Wg))
    layer.check(G, dz.T @ X, (r + 4 * k * U24) * rss(dz.T, X) + 1e-6 * rss(DY.T, X))
    assert np.all(np.abs(layer.f64(db) - dz.sum(0)) <= 8 * (1 + np.sqrt(k)) * U24 * np.abs(dz).sum(0) + 5e-7 * np.abs(DY).sum(0))
    assert int((dx != 0).any(1).sum()) <= k
    dx, Gg, Gu = qg.int8_gated_backward(dy, zg, zu, x, *wg, *wu)
    a, da = O.act(ZG, "silu")
    dzg, dzu = DY * ZU * da, DY * a
    layer.check(dx[at], dzg @ Wg + dzu @ Wu, (r + 4 * m * U24) * (rss(dzg, Wg) + rss(dzu, Wu)) + 1e-6 * (rss(DY * ZU, Wg) + rss(DY * ZG, Wu)))
    layer.check(Gg, dzg.T @ X, (r + 4 * k * U24) * rss(dzg.T, X) + 1e-6 * rss((DY * ZU).T, X))
    layer.check(Gu, dzu.T @ X, (r + 4 * k * U24) * rss(dzu.T, X) + 1e-6 * rss((DY * ZG).T, X))
    assert int((dx != 0).any(1).sum()) <= k
