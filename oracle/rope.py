"""Position rotation of queries and keys (rotary embedding).

Test infrastructure only (see the package docstring): the GPU path never
imports this module.

Pair i of a head's first R channels turns by positions * inv_freq[i]: the
plane rotation (x cos f - y sin f, y cos f + x sin f), evaluated here in
extended precision (long double angles).  Pairs are (i, i + R/2) or (2i, 2i+1);
channels from R on stay as they are.
"""

from __future__ import annotations

import numpy as np

TWO_PI = 2 * np.longdouble("3.14159265358979323846264338327950288")


def pair_channels(R: int, neighbours: bool):
    i = np.arange(R // 2)
    return (2 * i, 2 * i + 1) if neighbours else (i, i + R // 2)


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, neighbours: bool) -> np.ndarray:
    """x [T, heads, D] in fp64 -> rotated, fp64."""
    first, second = pair_channels(2 * len(inv_freq), neighbours)
    angle = np.asarray(positions).astype(np.longdouble)[:, None] * np.asarray(inv_freq, np.float64).astype(np.longdouble)
    angle = angle - np.rint(angle / TWO_PI) * TWO_PI
    c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
    y = np.array(x, np.float64)
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


def pair_sums(x: np.ndarray, R: int, neighbours: bool) -> np.ndarray:
    """|x| + |y| of each channel's pair (0 where nothing turns): what the rotation's rounding is relative to."""
    first, second = pair_channels(R, neighbours)
    out = np.zeros(x.shape)
    out[..., first] = out[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    return out
