"""Plain fp64 numpy reference of the operators around the INT8 linear layer: residual stream norms, the linear layer with
an epilogue (bias, activation, residual; gated pair), and the loss of a language model's head.  Inputs are decoded values
(float64 arrays); nothing is rounded."""
from __future__ import annotations

import math

import numpy as np


# ---------------------------------------------------------------- residual stream
def _inv_rms(v, eps):
    return 1.0 / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps)


def residual_norm_forward(h, y=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6):
    """Returns (h', u); gate: None, [d] or [tokens][d]."""
    if y is not None:
        n = y if w_post is None else w_post * y * _inv_rms(y, eps)
        h = h + scale * (1.0 if gate is None else gate) * n
    return h, None if w_pre is None else w_pre * h * _inv_rms(h, eps)


def residual_norm_backward(du, dh_next, h_next, y=None, w_post=None, gate=None, w_pre=None, scale=1.0, eps=1e-6):
    """Returns (dh, dy, dw_pre, dw_post, dgate), None for what has no input."""
    dh = np.zeros_like(h_next) if dh_next is None else dh_next
    dw_pre = dy = dw_post = dgate = None
    if du is not None:
        r = _inv_rms(h_next, eps)
        a = w_pre * du
        dh = dh + r * (a - h_next * r * r * np.mean(a * h_next, axis=1, keepdims=True))
        dw_pre = np.sum(du * h_next * r, axis=0)
    if y is not None:
        g = 1.0 if gate is None else gate
        dn = scale * g * dh
        if w_post is None:
            n, dy = y, dn * np.ones_like(y)
        else:
            q = _inv_rms(y, eps)
            n = w_post * y * q
            b = w_post * dn
            dy = q * (b - y * q * q * np.mean(b * y, axis=1, keepdims=True))
            dw_post = np.sum(dn * y * q, axis=0)
        if gate is not None:
            dgate = scale * dh * n
            if np.ndim(gate) == 1:
                dgate = dgate.sum(axis=0)
    return dh, dy, dw_pre, dw_post, dgate


# ---------------------------------------------------------------- linear layer with an epilogue
_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, kind):
    """(act(z), act'(z))"""
    if kind == "none":
        return z, np.ones_like(z)
    if kind == "relu":
        return np.maximum(z, 0.0), (z > 0).astype(np.float64)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return z * s, s + z * s * (1.0 - s)
    if kind == "gelu":
        cdf = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
        return z * cdf, cdf + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    raise ValueError(kind)


def linear_act_forward(x, W, bias=None, residual=None, kind="none"):
    """Returns (y, z): z = x W^T + bias, y = act(z) + residual."""
    z = x @ W.T
    if bias is not None:
        z = z + bias
    y = act(z, kind)[0]
    return (y if residual is None else y + residual), z


def linear_act_backward(dy, z, x, W, kind="none"):
    """Returns (dx, G, dbias)."""
    dz = dy if kind == "none" else dy * act(z, kind)[1]
    return dz @ W, dz.T @ x, dz.sum(axis=0)


def gated_forward(x, Wg, Wu, kind="silu"):
    """Returns (y, zg, zu): y = act(x Wg^T) * (x Wu^T)."""
    zg, zu = x @ Wg.T, x @ Wu.T
    return act(zg, kind)[0] * zu, zg, zu


def gated_backward(dy, zg, zu, x, Wg, Wu, kind="silu"):
    """Returns (dx, Gg, Gu)."""
    a, da = act(zg, kind)
    dzg, dzu = dy * zu * da, dy * a
    return dzg @ Wg + dzu @ Wu, dzg.T @ x, dzu.T @ x


# ---------------------------------------------------------------- loss of the head
def head_loss_forward(x, W, labels):
    """Returns (loss [T], lse [T]); a label outside [0, vocab) has loss 0."""
    logits = x @ W.T
    top = logits.max(axis=1)
    lse = top + np.log(np.exp(logits - top[:, None]).sum(axis=1))
    learned = (labels >= 0) & (labels < W.shape[0])
    at = np.where(learned, labels, 0)
    return np.where(learned, lse - logits[np.arange(len(labels)), at], 0.0), lse


def head_loss_backward(x, W, labels, dloss):
    """Returns (dx, dW) of sum_t dloss[t] loss[t]; rows of x without a loss are not used."""
    learned = (labels >= 0) & (labels < W.shape[0])
    x = np.where(learned[:, None], x, 0.0)
    logits = x @ W.T
    p = np.exp(logits - logits.max(axis=1, keepdims=True))
    p /= p.sum(axis=1, keepdims=True)
    p[np.arange(len(labels)), np.where(learned, labels, 0)] -= 1.0
    dl = np.where(learned, dloss, 0.0)[:, None] * p
    return dl @ W, dl.T @ x
