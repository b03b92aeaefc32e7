"""The fp64 reference of the operators around the linear layer: every gradient against central differences of its forward
pass, and the identities that pin the forward pass."""
import numpy as np
import pytest

from oracle import layers as O

G = np.random.default_rng(7)


def numeric(f, x, step=1e-6):
    """Gradient of the scalar f at x by central differences (error about step^2 times the third derivative)."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        down = f()
        x[i] = keep
        g[i] = (up - down) / (2 * step)
    return g


def close(a, b):
    assert np.linalg.norm(a - b) <= 1e-7 * max(1.0, np.linalg.norm(b))


@pytest.mark.parametrize("gate", [None, "channel", "token"])
@pytest.mark.parametrize("post", [False, True])
def test_residual_norm_gradients(gate, post):
    T, d, scale, eps = 3, 7, 0.7, 1e-3
    h, y = G.standard_normal((T, d)), G.standard_normal((T, d))
    w_pre, w_post = G.standard_normal(d), G.standard_normal(d) if post else None
    g = {None: None, "channel": G.standard_normal(d), "token": G.standard_normal((T, d))}[gate]
    cu, ch = G.standard_normal((T, d)), G.standard_normal((T, d))

    def f():
        hn, u = O.residual_norm_forward(h, y, w_post, g, w_pre, scale, eps)
        return np.sum(cu * u) + np.sum(ch * hn)

    hn, u = O.residual_norm_forward(h, y, w_post, g, w_pre, scale, eps)
    assert np.allclose(np.mean((u / w_pre) ** 2, axis=1), 1 - eps / (np.mean(hn * hn, axis=1) + eps))   # unit rms up to eps
    dh, dy, dw_pre, dw_post, dgate = O.residual_norm_backward(cu, ch, hn, y, w_post, g, w_pre, scale, eps)
    close(dh, numeric(f, h))
    close(dy, numeric(f, y))
    close(dw_pre, numeric(f, w_pre))
    if post:
        close(dw_post, numeric(f, w_post))
    else:
        assert dw_post is None
    if gate:
        close(dgate, numeric(f, g))
    else:
        assert dgate is None


@pytest.mark.parametrize("kind", ["none", "relu", "silu", "gelu"])
def test_linear_gradients(kind):
    T, m, n = 4, 5, 6
    x, W, b, r = (G.standard_normal(s) for s in ((T, n), (m, n), (m,), (T, m)))
    c = G.standard_normal((T, m))
    f = lambda: np.sum(c * O.linear_act_forward(x, W, b, r, kind)[0])
    y, z = O.linear_act_forward(x, W, b, r, kind)
    dx, gw, db = O.linear_act_backward(c, z, x, W, kind)
    close(dx, numeric(f, x))
    close(gw, numeric(f, W))
    close(db, numeric(f, b))
    close(c, numeric(f, r))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_gradients(kind):
    T, m, n = 4, 5, 6
    x, Wg, Wu, c = (G.standard_normal(s) for s in ((T, n), (m, n), (m, n), (T, m)))
    f = lambda: np.sum(c * O.gated_forward(x, Wg, Wu, kind)[0])
    _, zg, zu = O.gated_forward(x, Wg, Wu, kind)
    dx, gg, gu = O.gated_backward(c, zg, zu, x, Wg, Wu, kind)
    close(dx, numeric(f, x))
    close(gg, numeric(f, Wg))
    close(gu, numeric(f, Wu))


def test_head_loss_gradients():
    T, V, h = 5, 9, 4
    x, W, dloss = G.standard_normal((T, h)), G.standard_normal((V, h)), G.standard_normal(T)
    labels = np.array([0, 8, -100, 3, 9])            # first and last entry, two without a loss
    f = lambda: np.sum(dloss * O.head_loss_forward(x, W, labels)[0])
    loss, lse = O.head_loss_forward(x, W, labels)
    assert loss[2] == loss[4] == 0 and np.allclose(np.exp(x @ W.T - lse[:, None]).sum(axis=1), 1)
    dx, dW = O.head_loss_backward(x, W, labels, dloss)
    close(dx, numeric(f, x))
    close(dW, numeric(f, W))
    assert not dx[2].any() and not dx[4].any()


def test_head_loss_of_equal_logits_is_the_log_of_the_vocabulary():
    loss, _ = O.head_loss_forward(np.zeros((2, 3)), np.ones((11, 3)), np.array([0, 10]))
    assert np.allclose(loss, np.log(11))


def test_head_loss_ignores_what_rows_without_a_label_hold():
    x, W = G.standard_normal((3, 4)), G.standard_normal((6, 4))
    labels = np.array([2, -1, 5])
    clean = O.head_loss_backward(x, W, labels, np.ones(3))
    x[1] = np.nan
    for a, b in zip(clean, O.head_loss_backward(x, W, labels, np.ones(3))):
        assert np.array_equal(a, b)
