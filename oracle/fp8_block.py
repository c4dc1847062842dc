"""Plain NumPy definitions of the 8-bit block's operators: e4m3 rows and weights
with a scale for each 128, their product, and heads with positions.  Definitions
as include/acid.h states them; 64 bits but where a rounding to fp32 is part of the
definition (scales and the quotients that become codes)."""
from __future__ import annotations

import numpy as np

from .acid_oracle import gelu_tanh

GROUP = 128


def e4m3_values():
    """What the 256 codes stand for: sign, four bits of exponent (bias 7), three of
    fraction; 0x7f and 0xff are NaN, there are no infinities."""
    v = np.empty(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        v[c] = np.nan if c & 127 == 127 else f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        v[c] = -v[c] if c & 128 else v[c]
    return v


VALUES = e4m3_values()


def to_e4m3(x):
    """The e4m3 value nearest to each x, the one with an even code of two; past 448: 448."""
    x = np.asarray(x, np.float64)
    grid = VALUES[:127]                       # 0 .. 448, ascending: value i has code i
    a = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(grid, a)             # first value >= a
    lo = np.maximum(hi - 1, 0)
    up = grid[hi] - a
    down = a - grid[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.where(x < 0, -grid[code], grid[code])


def quantize(x):
    """(values of the codes, scales) of fp32 groups x [..., group] of finite numbers."""
    x = np.asarray(x, np.float32)
    most = np.abs(x).max(-1)
    scale = np.maximum(most / np.float32(448.0), np.float32(2.0 ** -126))
    inv = np.float32(1.0) / scale
    return to_e4m3(x * inv[..., None]), scale


def quantize_rows(x):
    """(code values [rows, k], scales [ceil(k/128), rows]) of fp32 rows."""
    x = np.asarray(x, np.float32)
    rows, k = x.shape
    codes, scales = np.empty((rows, k)), np.empty((-(-k // GROUP), rows), np.float32)
    for g in range(scales.shape[0]):
        at = slice(g * GROUP, (g + 1) * GROUP)
        codes[:, at], scales[g] = quantize(x[:, at])
    return codes, scales


def quantize_weight(w):
    """(code values [n, k], scales [ceil(n/128), ceil(k/128)]) of fp32 w [k, n]."""
    w = np.asarray(w, np.float32).T
    n, k = w.shape
    codes, scales = np.empty((n, k)), np.empty((-(-n // GROUP), -(-k // GROUP)), np.float32)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            at = (slice(i * GROUP, (i + 1) * GROUP), slice(j * GROUP, (j + 1) * GROUP))
            block, scales[i, j] = quantize(w[at].reshape(-1))
            codes[at] = block.reshape(w[at].shape)
    return codes, scales


def rows_values(codes, scales):
    """[rows, k] in 64 bits of code values and their scales [ceil(k/128), >= rows]."""
    codes = np.asarray(codes, np.float64)
    s = np.asarray(scales, np.float64)[:, :codes.shape[0]].T
    return codes * np.repeat(s, GROUP, 1)[:, :codes.shape[1]]


def weight_values(codes, scales):
    """[n, k] in 64 bits of a weight's code values and scales."""
    codes = np.asarray(codes, np.float64)
    s = np.repeat(np.repeat(np.asarray(scales, np.float64), GROUP, 0), GROUP, 1)
    return codes * s[:codes.shape[0], :codes.shape[1]]


def linear(a, w, bias=None, gelu=False, gate=None, residual=None):
    """a [m, k], w [n, k] in 64 bits: y = a w^T + bias, then GELU, or residual + gate y."""
    y = a @ w.T + (0.0 if bias is None else np.asarray(bias, np.float64))
    if gelu:
        return gelu_tanh(y)
    return y if gate is None else np.asarray(residual, np.float64) + np.asarray(gate, np.float64) * y


def ln_modulate(x, shift, scale, rows_per_mod=0, eps=1e-6):
    x = np.asarray(x, np.float64)
    row = np.arange(x.shape[0]) // (rows_per_mod or max(1, x.shape[0]))
    x = x - x.mean(1, keepdims=True)
    x = x / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    shift, scale = (np.atleast_2d(np.asarray(v, np.float64))[row] for v in (shift, scale))
    return x * (1 + scale) + shift


def heads(rows, n_heads, positions, freqs, sections, pairs="adjacent", norm="none", weight=None, bias=None,
          scale=1.0, eps=1e-6):
    """rows [tokens, n_heads * d] -> [n_heads, tokens, d]: norm, weight and bias, each pair
    turned by positions[axis] * freqs, all times scale."""
    x = np.asarray(rows, np.float64)
    tokens = x.shape[0]
    x = x.reshape(tokens, n_heads, -1)
    d = x.shape[2]
    if norm == "rms_row":
        x = x / np.sqrt((x * x).mean((1, 2), keepdims=True) + eps)
    elif norm != "none":
        if norm == "layer":
            x = x - x.mean(2, keepdims=True)
        x = x / np.sqrt((x * x).mean(2, keepdims=True) + eps)
    if weight is not None:
        x = x * np.asarray(weight, np.float64).reshape((n_heads, d) if norm == "rms_row" else (d,))
    if bias is not None:
        x = x + np.asarray(bias, np.float64)
    n = int(sum(sections))
    out = x.copy()
    i = 0
    for axis, count in enumerate(sections):
        for _ in range(count):
            t = np.asarray(positions[axis], np.float64) * float(freqs[i])
            p, q = (2 * i, 2 * i + 1) if pairs == "adjacent" else (i, n + i)
            u, v = x[:, :, p], x[:, :, q]
            out[:, :, p] = u * np.cos(t)[:, None] - v * np.sin(t)[:, None]
            out[:, :, q] = u * np.sin(t)[:, None] + v * np.cos(t)[:, None]
            i += 1
    return scale * out.transpose(1, 0, 2)
