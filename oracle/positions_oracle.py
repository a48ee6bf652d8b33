"""Plain fp64 oracle of include/apbv_positions.h, written from its definitions.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def rotate(x, positions, inv_freq, axis, adjacent=False, weight=None, eps=0.0):
    """Rows x [tokens, heads, d] float64, positions [axes, tokens], a frequency and an axis per pair -> rows, normed and turned, and
    for each element the sum of the absolute values of the two products that it is made of (for error bounds)."""
    x = np.asarray(x, np.float64)
    n, _, d = x.shape
    if weight is not None:
        x = x * np.asarray(weight, np.float64) / np.sqrt((x * x).sum(-1, keepdims=True) / d + eps)
    out, parts, half = x.copy(), np.abs(x), len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        for t in range(n):
            angle = float(positions[axis[i]][t]) * float(inv_freq[i])
            c, s = np.cos(angle), np.sin(angle)
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
            parts[t, :, a] = np.abs(x[t, :, a] * c) + np.abs(x[t, :, b] * s)
            parts[t, :, b] = np.abs(x[t, :, b] * c) + np.abs(x[t, :, a] * s)
    return out, parts
