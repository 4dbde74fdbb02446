"""Rotary positions of a chunk in float64 (test infrastructure only).  Written from the definition: the pair (a, b) of a row at position p is the
complex number a + ib, multiplied by m exp(i p f) on the way forward and by its conjugate on the way back."""
from __future__ import annotations

import math

import numpy as np


def positions_and_key_rows(segs):
    """Position and key row of every query row of the segment table [(q_start, q_len, kv_start, kv_len)]."""
    pos, key = [], []
    for _, n, kv0, kv in segs:
        pos += [kv - n + i for i in range(n)]
        key += [kv0 + kv - n + i for i in range(n)]
    return np.array(pos, dtype=np.int64), np.array(key, dtype=np.int64)


def pairs(rotary_dim, interleaved):
    j = np.arange(rotary_dim // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rotary_dim // 2)


def rotate(x, positions, frequencies, interleaved, magnitude=1.0, backward=False):
    """x [rows, heads, dim] float64 -> the rotated copy."""
    a, b = pairs(2 * len(frequencies), interleaved)
    turn = magnitude * np.exp(1j * np.outer(positions, frequencies))[:, None, :]
    z = (x[..., a] + 1j * x[..., b]) * (np.conj(turn) if backward else turn)
    y = x.copy()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def size(x, frequencies, interleaved, magnitude=1.0):
    """|a| + |b| of each element's pair times the magnitude, |x| for what is copied: what rounding errors are relative to."""
    a, b = pairs(2 * len(frequencies), interleaved)
    y = np.abs(x)
    y[..., a] = y[..., b] = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y


def frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0, original_length=0, low=1.0, high=32.0):
    out = []
    for j in range(rotary_dim // 2):
        b = base * factor ** (rotary_dim / (rotary_dim - 2)) if scaling == "base" else base
        f = 1.0 / b ** (2 * j / rotary_dim)
        if scaling == "linear":
            f = f / factor
        if scaling == "ramp":
            turns = original_length * f / (2 * math.pi)
            keep = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)
