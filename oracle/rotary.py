"""Rotary positions in extended precision.

Parity: pinned by hand-worked cases (tests/test_oracle_window.py). The paper has
no counterpart: its caches hold rows that are turned already.
"""
from __future__ import annotations

import numpy as np


def rotary(x, positions, freqs, interleaved=False, scale=1.0):
    """x [..., H, T, D] turned by positions [..., T] (broadcast over H): fp64.

    Angles are formed in long double: 2^31 turns of a position leave 1e-9."""
    x = np.asarray(x, np.float64)
    n = len(freqs)
    angle = np.asarray(positions).astype(np.longdouble)[..., None, :, None] * np.asarray(freqs, np.longdouble)
    cos, sin = np.cos(angle).astype(np.float64) * scale, np.sin(angle).astype(np.float64) * scale
    out = x.copy()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., first], x[..., second]
    out[..., first] = a * cos - b * sin
    out[..., second] = a * sin + b * cos
    return out
