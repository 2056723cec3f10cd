"""Oracle of the 8-bit integer projections: rows of codes with a scale each, and
the product with a scale for each token and output channel, from the definitions
(readings Q1-Q3; the paper's models run at their own precision, this is a
variant of F's projections):

  Q1 a row y has the scale s = fp32(max |y_i|) / 127 and the codes rint(y_i / s),
     fp32 quotients, ties to even; zeros: scale 0, codes 0; a NaN or an infinity:
     scale NaN, codes 0;
  Q2 behind RMSNorm y = x / sqrt(mean(x^2) + eps) * gain, behind the gate
     y = SiLU(gate) * up, neither rounded before Q1;
  Q3 Y = bf16(sum_k xq wq * (xs * ws) + R), the sum exact;
  Q4 a decoder layer with int8 projections is that of oracle.decoder with Q1-Q3 in
     place of its products: Q, K, V from the rows of the first norm, the output
     projection from the rows of the attention's bf16 output, gate and up (bf16)
     from the rows of the second norm, the down projection from Q2's rows.
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np

from . import attention, bf16_round, int8_read
from . import decoder as D


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


def decoder_layers(x: np.ndarray, layers, n_q_heads: int, n_kv_heads: int, head_dim: int, eps: float, theta: float,
                   kv_int8: bool) -> np.ndarray:
    """Q4 from position 0: layers as dicts of (codes, scales) in the [out][in] layout
    (wq, wk, wv, wo, w_gate_up, w_down) and the gains; ``kv_int8``: keys and values
    read back from an int8 cache.  bf16 where the layer stores."""
    n, pos = x.shape[0], np.arange(x.shape[0])
    for w in layers:
        h = quantize_rows(rmsnorm(x, w["g_attn"], eps))
        q, k, v = (bf16_round(product(*h, *w[name])) for name in ("wq", "wk", "wv"))
        q = bf16_round(D.rope(q.reshape(n, n_q_heads, head_dim), pos, theta))
        k = bf16_round(D.rope(k.reshape(n, n_kv_heads, head_dim), pos, theta))
        v = v.reshape(n, n_kv_heads, head_dim)
        if kv_int8:
            k, v = int8_read(k), int8_read(v)
        o = bf16_round(attention(q, k, v, 0, head_dim ** -0.5)).reshape(n, n_q_heads * head_dim)
        x = bf16_round(product(*quantize_rows(o), *w["wo"], x))
        gu = bf16_round(product(*quantize_rows(rmsnorm(x, w["g_mlp"], eps)), *w["w_gate_up"]))
        x = bf16_round(product(*quantize_rows(silu_mul(gu)), *w["w_down"], x))
    return x
