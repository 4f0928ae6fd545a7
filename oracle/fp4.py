"""OCP MXFP4 weights: E2M1 codes with one E8M0 scale for 32 of them, and the
linear layer with E4M3 activations.

Test infrastructure only (see the package docstring): the GPU path never
imports this module.  Written from the OCP Microscaling Formats specification:
E2M1 has one sign, two exponent and one fraction bit, bias 1, subnormals and no
infinity or NaN; E8M0 is 2^(byte - 127), 255 NaN.
"""

from __future__ import annotations

import numpy as np

from . import e4m3, quantize as q

GROUP = 32
E_MIN, E_MAX = -100, 125


def decode_table() -> np.ndarray:
    """Value of each of the 16 codes, fp64."""
    out = []
    for c in range(16):
        e, m = (c >> 1) & 3, c & 1
        mag = m * 0.5 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)
        out.append(-mag if c & 8 else mag)
    return np.array(out)


def encode(v: np.ndarray) -> np.ndarray:
    """fp64 values -> codes: the nearest of the 8 magnitudes, ties to the even code, 6 beyond."""
    grid = decode_table()[:8]
    mag = np.abs(v)
    mid = (grid[1:] + grid[:-1]) / 2
    up = np.searchsorted(mid, mag, side="left")           # mag == mid[i]: code i, which is even only where i is
    tie = (up < 7) & (mag == mid[np.minimum(up, 6)]) & (up % 2 == 1)
    code = up + tie
    return (code | (np.signbit(v).astype(np.int64) << 3)).astype(np.uint8)


def group_exponents(x_bits: np.ndarray) -> np.ndarray:
    """e of every group of 32 of bf16 rows [N, K]: the exponent of the largest magnitude rounded (ties to even) to two
    significant bits, less 2, in [-100, 125]."""
    x = np.abs(q.bf16_to_f32(x_bits).astype(np.float64))
    top = x.reshape(x.shape[0], -1, GROUP).max(-1)
    m, e = np.frexp(np.where(top > 0, top, 2.0 ** -140))  # top = m 2^e, 1/2 <= m < 1: steps of 1/4
    n = np.rint(m * 4)                                     # 2, 3, or 4 (the next power of two)
    return np.clip(np.where(n == 4, e, e - 1).astype(np.int64) - 2, E_MIN, E_MAX)


def quantize(x_bits: np.ndarray):
    """bf16 bits [N, K] -> (packed codes [N, K/2], scale bytes [N, K/32])."""
    e = group_exponents(x_bits)
    v = q.bf16_to_f32(x_bits).astype(np.float64) * 2.0 ** -np.repeat(e, GROUP, 1).astype(np.float64)
    c = encode(v)
    return (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8), (e + 127).astype(np.uint8)


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Weights [N, K] in fp64 (exact)."""
    tab = decode_table()
    v = np.stack((tab[codes & 15], tab[codes >> 4]), -1).reshape(codes.shape[0], -1)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, 1)[:, :v.shape[1]]


def gemm(a_codes: np.ndarray, sa, w: np.ndarray) -> np.ndarray:
    """dec(A) W^T * sa in fp64, W decoded [N, K]."""
    acc = e4m3.decode(a_codes) @ w.T
    sa = np.asarray(sa, np.float32).astype(np.float64)
    return acc * (sa.reshape(-1, 1) if sa.ndim else sa)


def error_bound(a_codes: np.ndarray, sa, w: np.ndarray) -> np.ndarray:
    """What the matrix cores' sums may be off by, as for E4M3 weights: each aligned group of 8 products within
    8 * 2^-13 of its largest, the fp32 accumulation of K/8 groups (and of a few partial sums) within 2^-24 each of all
    magnitudes; then two fp32 roundings of the scaled result."""
    a, b = np.abs(e4m3.decode(a_codes)), np.abs(w)
    M, K = a.shape
    N = b.shape[0]
    top = np.zeros((M, N))
    for k in range(0, K, 8):
        top += (a[:, None, k:k + 8] * b[None, :, k:k + 8]).max(-1)
    total = a @ b.T
    sa = np.asarray(sa, np.float32).astype(np.float64)
    sa = np.abs(sa.reshape(-1, 1) if sa.ndim else sa)
    return (8 * 2.0 ** -13 * top + (K / 8 + 32) * 2.0 ** -24 * total) * sa
