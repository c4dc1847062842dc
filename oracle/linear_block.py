"""Plain fp64 NumPy definitions of the linear-attention block's operators:
linear attention with per-head decay, the seam between two blocks, and 4-bit
weights with group scales.  Definitions as include/acid.h states them; no
chunking, no layouts but the documented ones."""
from __future__ import annotations

import numpy as np

from .acid_oracle import gelu_tanh


def linear_attention(q, k, v, slopes, state=None, scale=1.0):
    """q, k, v [heads, L, d], slopes [heads], state [heads, d, d] or None.
    Returns (o [L, heads*d], state): S = exp(-slope) S + k^T v, o = scale q S,
    one token after the other."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    heads, L, d = q.shape
    lam = np.exp(-np.asarray(slopes, np.float64))[:, None, None]
    S = np.zeros((heads, d, d)) if state is None else np.array(state, np.float64)
    o = np.zeros((L, heads, d))
    for t in range(L):
        S = lam * S + k[:, t, :, None] * v[:, t, None, :]
        o[t] = scale * (q[:, t, None, :] @ S)[:, 0]
    return o.reshape(L, heads * d), S


def norm(x, kind, eps):
    x = np.asarray(x, np.float64)
    if kind == "layer":
        x = x - x.mean(1, keepdims=True)
    if kind != "none":
        x = x / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    return x


def residual_norm(h, y=None, res_scale=1.0, post="none", post_weight=None, gate=None,
                  pre="layer", pre_weight=None, shift=None, scale=None, rows_per_mod=0,
                  eps=1e-6):
    """(h', out) of the seam between two blocks."""
    h = np.asarray(h, np.float64)
    row = np.arange(h.shape[0]) // (rows_per_mod or max(h.shape[0], 1))

    def vec(m, default):  # modulation rows spread over the rows
        return default if m is None else np.atleast_2d(np.asarray(m, np.float64))[row]

    def weight(w):
        return 1.0 if w is None else np.asarray(w, np.float64)

    if y is not None:
        h = res_scale * h + vec(gate, 1.0) * norm(y, post, eps) * weight(post_weight)
    out = norm(h, pre, eps) * weight(pre_weight) * (1.0 + vec(scale, 0.0)) + vec(shift, 0.0)
    return h, out


def w4_quantize(w, group):
    """fp32 [K, N] -> (codes 0..15 [N, K], scales fp32 [N, K/group])."""
    w = np.ascontiguousarray(np.asarray(w, np.float32).T)
    N, K = w.shape
    g = w.reshape(N, K // group, group)
    most = np.abs(g).max(2)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        scales = (most / np.float32(7)).astype(np.float32)
        scales[~np.isfinite(g).all(2)] = np.nan
        c = np.rint(g / scales[:, :, None])
    c = np.where(scales[:, :, None] > 0, np.clip(c, -8, 7), 0.0) + 8
    return c.reshape(N, K).astype(np.uint8), scales


def _place(N, K):
    """(tile, block, run, byte, shift) of each [N, K] code in the layout."""
    n, k = np.arange(N)[:, None], np.arange(K)[None, :]
    e = k % 8
    nibble = e // 2 + 4 * (e % 2)
    return (n // 16 + 0 * k, k // 128 + 0 * n, 16 * (k // 8 % 4) + n % 16,
            4 * (k // 32 % 4) + nibble // 2 + 0 * n, 4 * (nibble % 2) + 0 * n)


def w4_pack(codes, scales):
    """Codes [N, K] and scales [N, K/group] in the library's layout; outputs
    past N have code 8 and scale 0."""
    N, K = codes.shape
    tiles = -(-N // 16)
    full = np.full((tiles * 16, K), 8, np.uint8)
    full[:N] = codes
    out = np.zeros((tiles, K // 128, 64, 16), np.uint8)
    tile, block, run, byte, shift = _place(tiles * 16, K)
    np.bitwise_or.at(out, (tile, block, run, byte), full << shift)
    s = np.zeros((tiles * 16, scales.shape[1]), np.float32)
    s[:N] = scales
    return out, np.ascontiguousarray(s.reshape(tiles, 16, -1).transpose(0, 2, 1))


def w4_weights(codes, scales, N):
    """fp64 weights [N, K] of the library's layout."""
    K = codes.shape[1] * 128
    tile, block, run, byte, shift = _place(N, K)
    c = (codes[tile, block, run, byte] >> shift) & 15
    s = np.asarray(scales, np.float64).transpose(0, 2, 1).reshape(-1, scales.shape[1])[:N]
    return (c.astype(np.float64) - 8) * np.repeat(s, K // scales.shape[1], 1)


def linear_w4(x, codes, scales, N, bias=None, gelu=False):
    y = np.asarray(x, np.float64) @ w4_weights(codes, scales, N).T
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return gelu_tanh(y) if gelu else y
