"""Root-mean-square norm with the residual's addition and an E4M3 output.

Test infrastructure only (see the package docstring): the GPU path never
imports this module.

For every row: h = x + residual, y = h * w / sqrt(mean(h^2) + eps), the norm of
the Llama-family target (§4), in fp64 from bf16 inputs; h is stored as bf16 for
the next residual (h itself is the fp32 sum of two bf16 values, whose rounding
to bf16 is reproduced exactly here), y as bf16 and as E4M3 codes with a row's
or a given scale (§3.2 FP8 Post-Training Quantization).
"""

from __future__ import annotations

import numpy as np

from . import quantize as q


def residual_sum(x_bits: np.ndarray, residual_bits: np.ndarray = None) -> np.ndarray:
    """h in fp64: the fp32 sum of two bf16 values (the values themselves without a residual)."""
    x = q.bf16_to_f32(x_bits)
    if residual_bits is None:
        return x.astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        return (x + q.bf16_to_f32(residual_bits)).astype(np.float64)


def rms_norm(h: np.ndarray, weight_bits: np.ndarray, eps: float) -> np.ndarray:
    """y in fp64; a row that holds an infinity or a NaN is NaN throughout."""
    w = q.bf16_to_f32(weight_bits).astype(np.float64)
    ok = np.isfinite(h).all(axis=1, keepdims=True)
    h = np.where(ok, h, np.nan)
    return h * w / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + float(np.float32(eps)))


def row_scale(y: np.ndarray) -> np.ndarray:
    """max|y| / 448, at least 2^-100, in fp64 (2^-100 for a row of NaN)."""
    top = np.max(np.where(np.isfinite(y), np.abs(y), 0.0), axis=1)
    return np.maximum(top / 448.0, 2.0 ** -100)
