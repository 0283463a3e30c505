"""Reference of the 8-bit block operators and of group norm, in 64 bits (numpy, from the definitions)."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
ACT_NONE, ACT_RELU, ACT_RELU6, ACT_GELU, ACT_SILU = range(5)
_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(v, kind):
    v = np.asarray(v, np.float64)
    if kind == ACT_RELU:
        return np.maximum(v, 0.0)
    if kind == ACT_RELU6:
        return np.clip(v, 0.0, 6.0)
    if kind == ACT_GELU:
        return 0.5 * v * (1.0 + _erf(v / math.sqrt(2.0)))
    if kind == ACT_SILU:
        with np.errstate(over="ignore"):
            return v / (1.0 + np.exp(-v))
    return v


def e4m3(v):
    """The e4m3 value nearest to v, ties to even; |v| up to 448 (NaN stays NaN)."""
    v = np.asarray(v, np.float64)
    mag = np.maximum(np.abs(v), 2.0 ** -6)
    step = 2.0 ** (np.floor(np.log2(np.where(np.isfinite(mag), mag, 1.0))) - 3)
    return np.where(np.isfinite(v), np.round(v / step) * step, np.nan)


def quantize(x, group):
    """x [batch, rows, cols] (float32 values) -> (values [batch, rows, kp], scales [batch, kb, row blocks]).

    A scale is rounded once, to float32, and so is a value, x * 448 / largest to e4m3, so this is bit for bit: a quotient of float32
    numbers that is no midpoint of e4m3 is further from one than a rounding in 64 bits."""
    x = np.asarray(x, np.float32)
    batch, rows, cols = x.shape
    kb, rb = -(-cols // BLOCK), -(-rows // group)
    q = np.zeros((batch, rows, kb * BLOCK))
    scale = np.zeros((batch, kb, rb), np.float32)
    f32 = np.float32
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for i in range(batch):
            for r in range(rb):
                for b in range(kb):
                    cut = (i, slice(r * group, (r + 1) * group), slice(b * BLOCK, min((b + 1) * BLOCK, cols)))
                    top = np.max(np.abs(x[cut]))  # (numpy's max is NaN where one is)
                    top = f32(2.0 ** -100) if top < f32(2.0 ** -100) else top
                    scale[i, b, r] = top / f32(448.0)
                    q[cut] = e4m3(x[cut].astype(np.float64) * 448.0 / np.float64(top))
    return q, scale


def dequantize(q, scale, group):
    """[batch, rows, kp] in 64 bits."""
    q, scale = np.asarray(q, np.float64), np.asarray(scale, np.float64)
    rows = q.shape[1]
    wide = np.repeat(scale, group, axis=2)[:, :, :rows].transpose(0, 2, 1)
    return q * np.repeat(wide, BLOCK, axis=2)


def product(a, a_scale, b, b_scale, b_rows):
    """(a b^T, sum of the absolute products) of two batches in blocks, [batch, m, n]."""
    x, w = dequantize(a, a_scale, 1), dequantize(b, b_scale, b_rows)
    return x @ w.transpose(0, 2, 1), np.abs(x) @ np.abs(w).transpose(0, 2, 1)


def group_norm(x, gamma, beta, groups, kind, eps):
    """(y, values before the activation, 1 / sqrt(var + eps) per channel, mean per channel) of x [n, h, w, c]."""
    x = np.asarray(x, np.float64)
    n, h, w, c = x.shape
    parts = x.reshape(n, h * w, groups, c // groups)
    mean = parts.mean(axis=(1, 3), keepdims=True)
    rstd = 1.0 / np.sqrt(((parts - mean) ** 2).mean(axis=(1, 3), keepdims=True) + eps)
    v = ((parts - mean) * rstd).reshape(n, h, w, c)
    if gamma is not None:
        v = v * np.asarray(gamma, np.float64)
    if beta is not None:
        v = v + np.asarray(beta, np.float64)
    spread = lambda s: np.broadcast_to(s, parts.shape).reshape(n, h, w, c)  # noqa: E731
    return act(v, kind), v, spread(rstd), spread(mean)
