"""Norms around a block with gate and residual scale in float64 (test infrastructure only).  Next to each result stands the sum of the magnitudes
of the terms it is formed from, which is what float32 rounding errors are relative to."""
from __future__ import annotations

import numpy as np


def act(g, kind):
    """The gate's value and slope."""
    if kind == "plain":
        return g, np.ones_like(g)
    p = 1.0 / (1.0 + np.exp(-g))
    return (p, p * (1 - p)) if kind == "sigmoid" else (g * p, p + g * p * (1 - p))


def _inv(x, eps):
    return 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def forward(y, gate, residual, post, pre, eps, kind, alpha, beta):
    """{"out", "h"} and their sizes."""
    block = size = 0.0
    if y is not None:
        block = beta * (y * _inv(y, eps) * post if post is not None else y)
        if gate is not None:
            block = block * act(gate, kind)[0]
        size = np.abs(block)
    if residual is not None:
        block = block + alpha * residual
        size = size + np.abs(alpha * residual)
    out, sizes = {"out": block}, {"out": size}
    if pre is not None:
        out["h"], sizes["h"] = block * _inv(block, eps) * pre, size * _inv(block, eps) * np.abs(pre)
    return out, sizes


def _norm_back(x, w, d, eps):
    """Gradients of N(x; w) = x w / rms(x) for the gradient d of its result, with sizes: (dx, size, rows' dw, size)."""
    inv = _inv(x, eps)
    n = x * inv
    dx = inv * (d * w - n * (d * w * n).mean(-1, keepdims=True))
    size = inv * (np.abs(d * w) + np.abs(n) * np.abs(d * w * n).mean(-1, keepdims=True))
    return dx, size, d * n, np.abs(d * n)


def backward(y, gate, stored, post, pre, d_out, d_h, eps, kind, alpha, beta):
    """{"dy", "d_gate", "d_residual", "d_post", "d_pre"} and their sizes."""
    out, sizes = {}, {}
    t = size_t = 0.0
    if d_out is not None:
        t, size_t = d_out, np.abs(d_out)
    if pre is not None:
        dx, s, dw, sw = _norm_back(stored, pre, d_h, eps)
        t, size_t = t + dx, size_t + s
        out["d_pre"], sizes["d_pre"] = dw.sum(0), sw.sum(0)
    out["d_residual"], sizes["d_residual"] = alpha * t, abs(alpha) * size_t
    if y is None:
        return out, sizes
    u, size_u = beta * t, abs(beta) * size_t
    if gate is not None:
        a, slope = act(gate, kind)
        n = y * _inv(y, eps) * post if post is not None else y
        out["d_gate"], sizes["d_gate"] = u * n * slope, size_u * np.abs(n) * (np.abs(slope) + np.abs(gate * slope) + 1.0)
        u, size_u = u * a, size_u * np.abs(a)
    if post is not None:
        out["dy"], _, dw, _ = _norm_back(y, post, u, eps)
        _, sizes["dy"], _, sw = _norm_back(y, post, size_u, eps)
        out["d_post"], sizes["d_post"] = dw.sum(0), sw.sum(0)
    else:
        out["dy"], sizes["dy"] = u, size_u
    return out, sizes
