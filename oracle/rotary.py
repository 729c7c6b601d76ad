"""Rotary positions in plain numpy, 64 bits: the definitions of include/uzip_rotary.h."""
from __future__ import annotations

import numpy as np


def positions(lens, q_start, rows: int) -> np.ndarray:
    out = np.full(rows, -1, np.int32)
    for i in range(len(lens)):
        a, b = int(q_start[i]), int(q_start[i + 1])
        for r in range(a, min(b, rows)):
            out[r] = max(int(lens[i]) - (b - a) + (r - a), -1)
    return out


def pairs(rot: int, first: int, interleaved: bool):
    """The channels of each pair."""
    i = np.arange(rot // 2)
    return (first + 2 * i, first + 2 * i + 1) if interleaved else (first + i, first + rot // 2 + i)


def rotate(x, places, freq, interleaved: bool = False, first: int = 0, magnitude: float = 1.0, inverse: bool = False) -> np.ndarray:
    """x [rows, heads, dim]."""
    x = np.asarray(x, dtype=np.float64)
    freq = np.asarray(freq, dtype=np.float64)
    angle = np.asarray(places, dtype=np.float64)[:, None, None] * freq * (-1.0 if inverse else 1.0)
    a, b = pairs(2 * len(freq), first, interleaved)
    y = x.copy()
    y[..., a] = magnitude * (x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle))
    y[..., b] = magnitude * (x[..., a] * np.sin(angle) + x[..., b] * np.cos(angle))
    return y


def error(x, places, freq, interleaved: bool = False, first: int = 0, magnitude: float = 1.0) -> np.ndarray:
    """A bound on a turned value's error in 32 bits before it is rounded.  A cosine is off by the rest of its angle's
    rounding (|rest| <= pi / 4: 2^-24), its series (2^-28) and the series' and the magnitude's roundings (3 of
    2^-24 at most), the product with it by one more and the sum by one: 6 of 2^-24 of |a| + |b|.  The angle itself, a
    product of 55 bits and one with 2 / pi in 53: 2^-51 of its size."""
    x = np.abs(np.asarray(x, dtype=np.float64))
    angle = np.abs(np.asarray(places, dtype=np.float64))[:, None, None] * np.abs(np.asarray(freq, dtype=np.float64))
    a, b = pairs(2 * len(freq), first, interleaved)
    tol = np.zeros_like(x)
    tol[..., a] = tol[..., b] = (x[..., a] + x[..., b]) * abs(magnitude) * (6 * 2.0 ** -24 + 2.0 ** -51 * angle)
    return tol
