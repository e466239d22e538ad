"""CPU fp64 oracle of rotary positions — TEST INFRASTRUCTURE ONLY.

A head's first r dims form r / 2 pairs, (i, i + r / 2) or (2 i, 2 i + 1).  Pair i of the token at position p is turned by
p * f_i radians and multiplied by the magnitude; the other dims stay.  The paper names no positional term, so the
convention is pinned by its own properties only (closed forms, relative positions, adjointness).
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(r, base=10000.0, factor=1.0, original_len=0, low_turns=1.0, high_turns=32.0):
    """f_i = base^(-2 i / r), divided by `factor` where the pair makes few turns over the original context."""
    out = np.empty(r // 2)
    for i in range(r // 2):
        f = base ** (-2.0 * i / r)
        if original_len == 0:
            out[i] = f / factor
            continue
        g = (original_len * f / (2.0 * math.pi) - low_turns) / (high_turns - low_turns)
        g = min(1.0, max(0.0, g))
        out[i] = (1.0 - g) * f / factor + g * f
    return out


def rotate(x, positions, freq, interleaved=False, magnitude=1.0, grad=False):
    """x float64 [T, H, d] turned by positions [T]; grad: the transpose."""
    x = np.asarray(x, dtype=np.float64)
    out = x.copy()
    half = len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = np.asarray(positions, dtype=np.float64) * freq[i] * (-1.0 if grad else 1.0)
        c, s = magnitude * np.cos(angle)[:, None], magnitude * np.sin(angle)[:, None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out
