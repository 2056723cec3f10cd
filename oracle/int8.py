"""Oracle of the 8-bit integer projections: rows of codes with a scale each, and
the product with a scale for each token and output channel, from the definitions
(readings Q1-Q3; the paper's models run at their own precision, this is a
variant of F's projections):

  Q1 a row y has the scale s = fp32(max |y_i|) / 127 and the codes rint(y_i / s),
     fp32 quotients, ties to even; zeros: scale 0, codes 0; a NaN or an infinity:
     scale NaN, codes 0;
  Q2 behind RMSNorm y = x / sqrt(mean(x^2) + eps) * gain, behind the gate
     y = SiLU(gate) * up, neither rounded before Q1;
  Q3 Y = bf16(sum_k xq wq * (xs * ws) + R), the sum exact.
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np


def quantize_rows(y: np.ndarray) -> Tuple[np.ndarray, np.ndarray]:
    """Q1 of fp32 values: int64 codes [m, k], fp32 scales [m]."""
    y = np.asarray(y, dtype=np.float32)
    top = np.abs(y).max(-1)
    bad = ~np.isfinite(y).all(-1)
    s = np.where(bad, np.float32(np.nan), top / np.float32(127)).astype(np.float32)
    ok = (s > 0)
    with np.errstate(invalid="ignore"):
        codes = np.rint(y / np.where(ok, s, np.float32(1))[:, None])
    codes = np.where(ok[:, None], codes, 0)
    return np.clip(codes, -127, 127).astype(np.int64), s


def rmsnorm(x: np.ndarray, gain: np.ndarray, eps: float) -> np.ndarray:
    """Q2, fp64."""
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def silu_mul(gate_up: np.ndarray) -> np.ndarray:
    """Q2, fp64."""
    gate, up = np.split(gate_up, 2, -1)
    return gate / (1 + np.exp(-gate)) * up


def product(xq: np.ndarray, xs: np.ndarray, wq: np.ndarray, ws: np.ndarray, r: Optional[np.ndarray] = None) -> np.ndarray:
    """Q3 before its rounding, fp64."""
    y = (xq.astype(np.float64) @ wq.astype(np.float64).T) * (xs.astype(np.float64)[:, None] * ws.astype(np.float64))
    return y if r is None else y + r
