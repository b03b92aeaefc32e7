"""Attention half of a decoder layer in fp64: rotary positions, attention of one head over one sequence with its gradients, and a cache in
pages.  Written from the formulas, one head or one token at a time; numpy only."""
from __future__ import annotations

import numpy as np


def rope(x, positions, freqs, layout="half", amplitude=1.0, backward=False):
    """x [tokens][heads][d]: pairs of the first 2 len(freqs) elements turned by positions[token] * freqs[pair]."""
    y = np.array(x, dtype=np.float64)
    half = len(freqs)
    for t, p in enumerate(positions):
        angle = (float(p) * np.asarray(freqs, dtype=np.float64)) * (-1 if backward else 1)
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        a, b = np.array(x[t, :, first], dtype=np.float64), np.array(x[t, :, second], dtype=np.float64)
        y[t, :, first], y[t, :, second] = a * c - b * s, a * s + b * c
    return y


def rope_frequencies(rot, base=10000.0, factor=1.0, context=0, low=1.0, high=4.0):
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        turns = context * f / (2 * np.pi)
        keep = min(1.0, max(0.0, (turns - low) / (high - low))) if context > 0 else 0.0
        out.append(f * keep + f / factor * (1 - keep))
    return np.array(out)


def visible(n_q, n_k, causal=True, window=0, prefix=0):
    """bool [n_q][n_k]; query i stands at position i + n_k - n_q."""
    p, j = np.arange(n_q)[:, None] + n_k - n_q, np.arange(n_k)[None]
    if not causal:
        return np.ones((n_q, n_k), dtype=bool)
    return (j < prefix) | ((j <= p) & ((p - j < window) | (window == 0)))


def scores(q, k, scale, cap=0.0, slope=0.0):
    """(x, dx/draw): the scores of one head and their derivative by scale * q.k."""
    raw = scale * (q @ k.T)
    t = np.tanh(raw / cap) if cap > 0 else None
    x = raw if t is None else cap * t
    p = np.arange(len(q))[:, None] + len(k) - len(q)
    return x - slope * np.abs(p - np.arange(len(k))[None]), np.ones_like(raw) if t is None else 1 - t * t


def attention(q, k, v, scale, seen, cap=0.0, slope=0.0):
    """One head of one sequence: (o, lse, p); a row that sees nothing has o = 0, lse = -inf, p = 0."""
    x, _ = scores(q, k, scale, cap, slope)
    x = np.where(seen, x, -np.inf)
    top = x.max(axis=1, initial=-np.inf, keepdims=True)
    top = np.where(np.isinf(top), 0.0, top)
    e = np.exp(x - top)
    total = e.sum(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + top)[:, 0]
    p = np.where(total > 0, e / np.where(total > 0, total, 1.0), 0.0)
    return p @ v, lse, p


def attention_gradients(do, q, k, v, scale, seen, cap=0.0, slope=0.0, o=None):
    """(dq, dk, dv, ds) of one head; o: the output that delta = sum do o is formed with (None: the exact one)."""
    out, _, p = attention(q, k, v, scale, seen, cap, slope)
    _, factor = scores(q, k, scale, cap, slope)
    delta = (do * (out if o is None else o)).sum(axis=1, keepdims=True)
    ds = p * (do @ v.T - delta) * factor * scale
    return ds @ k, ds.T @ q, p.T @ do, ds


def cache_place(table, sequence, position, page_size, pages):
    """(page, row) of a position, None where it has no page."""
    if not 0 <= sequence < len(table) or not 0 <= position < len(table[sequence]) * page_size:
        return None
    page = int(table[sequence][position // page_size])
    return (page, position % page_size) if 0 <= page < pages else None


def paged_rows(table, sequence, length, page_size, pages, window=0):
    """Places of the visible positions of a sequence, and those positions."""
    end = min(max(int(length), 0), len(table[sequence]) * page_size)
    where = [(j, cache_place(table, sequence, j, page_size, pages)) for j in range(max(0, end - window) if window else 0, end)]
    return [(j, at) for j, at in where if at is not None], end
