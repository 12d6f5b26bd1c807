"""The operators between a block's products, and the dense int8 product, in plain
numpy: from their definitions in 64 bits, and step by step in the precision that
the interface states (fp32 operations, means and roots in fp64), which fixes every
bit of a norm's result.  It shares no code with the library."""
from __future__ import annotations

import math

import numpy as np

from . import formats as F

U = 2.0 ** -24  # half an fp32 step, relative


def _f64(a):
    return None if a is None else np.asarray(a, np.float64)


def norm64(v, weight, bias, eps, layer):
    v = _f64(v)
    if layer:
        v = v - v.mean(-1, keepdims=True)
    n = v / np.sqrt(np.mean(v * v, -1, keepdims=True) + eps) * _f64(weight)
    return n if bias is None else n + _f64(bias)


def stream64(residual, y, gate, scale, post_weight=None, post_bias=None, post_eps=1e-6, layer=False):
    u = _f64(y) if post_weight is None else norm64(y, post_weight, post_bias, post_eps, layer)
    return _f64(residual) + u * (1.0 if gate is None else _f64(gate)) * scale


def norm_steps(v, weight, bias, eps, layer):
    v = np.asarray(v, np.float32)
    d = v.astype(np.float64)
    if layer:
        d = d - d.mean(-1, keepdims=True)
    root = (1.0 / np.sqrt(np.mean(d * d, -1, keepdims=True) + eps)).astype(np.float32)
    n = d.astype(np.float32) * root * np.asarray(weight, np.float32)
    return n if bias is None else n + np.asarray(bias, np.float32)


def stream_steps(residual, y, gate, scale, post_weight=None, post_bias=None, post_eps=1e-6, layer=False):
    u = np.asarray(y, np.float32) if post_weight is None else norm_steps(y, post_weight, post_bias, post_eps, layer)
    t = u if gate is None else u * np.asarray(gate, np.float32)
    return np.asarray(residual, np.float32) + t * np.float32(scale)


def codes_steps(rows, kind):
    """The 8-bit codes (as bytes) and scales of fp32 rows."""
    rows = np.asarray(rows, np.float32)
    qmax = np.float32(127 if kind == "int8" else 448)
    codes, scales = np.zeros(rows.shape, np.uint8), np.zeros(rows.shape[0], np.float32)
    for m, v in enumerate(rows):
        if not np.isfinite(v).all():
            scales[m] = np.nan if np.isnan(v).any() else np.inf
            continue
        a = np.abs(v).max() if v.size else np.float32(0)
        scales[m] = a / qmax
        if a == 0:
            continue
        if a < np.float32(2.0 ** -118):
            v, a = v * np.float32(2.0 ** 60), a * np.float32(2.0 ** 60)
        t = v * (np.float32(1) / a * qmax)
        codes[m] = F.int_rne_clamp(t, 127).astype(np.int8).view(np.uint8) if kind == "int8" else F.e4m3_encode(np.clip(t, -448, 448))
    return codes, scales


def activation64(x, act, gated):
    x = _f64(x)
    g, u = (x[:, : x.shape[1] // 2], x[:, x.shape[1] // 2:]) if gated else (x, 1.0)
    with np.errstate(over="ignore", invalid="ignore"):
        if act == "silu":
            h = g / (1 + np.exp(-g))
        elif act == "gelu":
            # 0.5 g (1 + tanh z) with (1 + tanh z) / 2 = 1 / (1 + exp(-2 z)), which loses nothing where tanh z is near -1
            h = g / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
        else:
            h = np.maximum(g, 0)
        return h * u


def product64(xq, s_x, wq, s_w, bias=None):
    """Y in 64 bits from the exact integer sums, and the sums."""
    total = np.asarray(xq, np.int8).astype(np.int64) @ np.asarray(wq, np.int8).astype(np.int64).T
    y = total * _f64(s_x)[:, None] * _f64(s_w)
    return (y if bias is None else y + _f64(bias)), total
