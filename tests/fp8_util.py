"""Inputs and layouts of the 8-bit block's tests."""
import numpy as np
import torch

E4M3 = torch.float8_e4m3fn
U32 = 2.0 ** -24   # half a step of fp32, relative
U16 = 2.0 ** -8    # of bf16


def f64(t):
    return t.detach().double().cpu().numpy()


def normal(shape, seed, std=1.0, mean=0.0, dtype=torch.float32):
    x = np.random.default_rng(list(np.atleast_1d(seed))).standard_normal(shape, dtype=np.float32)
    return (torch.from_numpy(x) * std + mean).to(dtype).cuda()


def strided(rows, cols, dtype, pad=0, fill=0, multiple=1):
    """A [rows, cols] view of a matrix that is `pad` columns and up to a multiple wider, full
    of `fill`, and that matrix."""
    wide = -(-(cols + pad) // multiple) * multiple
    whole = torch.full((rows, wide), fill, device="cuda").to(dtype)
    return whole[:, :cols], whole


def fp8_rows(P, rows, k, pad=0, fill=0.0):
    """codes and scales as fp8_shapes has them, row-strided where pad is given."""
    cs, ss = P.fp8_shapes(rows, k)
    codes = strided(*cs, E4M3, pad, fill, 16)[0]
    scales = strided(*ss, torch.float32, 4 * (pad // 4), fill, 4)[0]
    return codes, scales


def quantized_rows(P, x):
    codes, scales = fp8_rows(P, *x.shape)
    P.quantize_fp8(x, codes, scales)
    return codes, scales


def quantized_weight(P, w):
    cs, ss = P.fp8_weight_shapes(w.shape[1], w.shape[0])
    codes, scales = torch.zeros(cs, dtype=E4M3, device="cuda"), torch.zeros(ss, device="cuda")
    P.quantize_fp8_weight(w, codes, scales)
    return codes, scales
