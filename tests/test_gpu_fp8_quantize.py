"""Rows and weights into e4m3, bit for bit against the definition; LN-modulated
rows within the roundings that it allows."""
import numpy as np
import pytest
import torch

from fp8_util import E4M3, f64, fp8_rows, normal, quantized_weight, strided
from gpu_util import assert_elementwise, need_gpu
from oracle import fp8_block as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROWS = [(1, 16), (1, 128), (3, 144), (4, 1040), (31, 112), (32, 256), (33, 272), (77, 1536), (129, 4112), (1000, 48)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,k", ROWS)
def test_rows(rows, k, dtype):
    P = need_gpu()
    x = normal((rows, k), [rows, k], 2.0, 0.1, dtype)
    x[0, 0], x[-1, -1] = 300.0, -1e-30
    if rows > 2:
        x[1] = 0
        x[2] *= 1e-38          # sums of tiny values: the smallest scale
    codes, scales = fp8_rows(P, rows, k, fill=3.0)
    P.quantize_fp8(x, codes, scales)
    want, ws = B.quantize_rows(x.float().cpu().numpy())
    assert np.array_equal(f64(scales)[:, :rows], ws.astype(np.float64))
    assert np.array_equal(f64(codes), want)
    assert (scales[:, rows:] == 3.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_strided_rows(dtype):
    P = need_gpu()
    x, _ = strided(45, 400, dtype, 24, multiple=8)
    x.copy_(normal((45, 400), 3, dtype=dtype))
    codes, whole = strided(45, 400, E4M3, 40, 1.5, 16)
    scales, swhole = strided(4, 48, F32, 8, 7.0, 4)
    P.quantize_fp8(x, codes, scales)
    want, ws = B.quantize_rows(x.float().cpu().numpy())
    assert np.array_equal(f64(codes), want) and np.array_equal(f64(scales)[:, :45], ws.astype(np.float64))
    assert (whole[:, 400:].float() == 1.5).all() and (swhole[:, 48:] == 7.0).all() and (swhole[:, 45:48] == 7.0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_spoils_its_group_alone(bad):
    P = need_gpu()
    x = normal((6, 304), 4)
    clean = fp8_rows(P, 6, 304)
    P.quantize_fp8(x, *clean)
    x[2, 130] = bad
    codes, scales = fp8_rows(P, 6, 304)
    P.quantize_fp8(x, codes, scales)
    assert torch.isnan(scales[1, 2]) and torch.isnan(scales).sum() == 1
    keep = torch.ones(6, 304, dtype=torch.bool, device="cuda")
    keep[2, 128:256] = False
    assert torch.equal(codes.float()[keep], clean[0].float()[keep])
    w = normal((304, 200), 5)
    w[140, 3] = bad
    _, ws = quantized_weight(P, w)
    assert torch.isnan(ws[0, 1]) and torch.isnan(ws).sum() == 1
    shift, scale = normal(304, 6), normal(304, 7)
    x = normal((6, 304), 8)
    x[2, 130] = bad  # the row's mean: all of its groups
    codes, scales = fp8_rows(P, 6, 304)
    P.ln_modulate_fp8(x, shift, scale, codes, scales)
    assert torch.isnan(scales[:, 2]).all() and torch.isnan(scales).sum() == 3


@pytest.mark.parametrize("n,k", [(1, 16), (16, 128), (127, 48), (128, 144), (129, 112), (257, 1040), (300, 272), (1000, 640)])
def test_weight(n, k):
    P = need_gpu()
    w = normal((k, n), [n, k], 0.02)
    w[0, 0], w[-1, -1] = 3.0, -2.0
    codes, scales = quantized_weight(P, w)
    want, ws = B.quantize_weight(w.cpu().numpy())
    assert np.array_equal(f64(scales), ws.astype(np.float64)) and np.array_equal(f64(codes), want)


@pytest.mark.parametrize("rows,hidden,mod", [(1, 16, 0), (2, 128, 1), (5, 144, 2), (7, 4096, 3), (33, 1536, 0), (6, 2048, 0),
                                             (9, 2064, 4), (3, 8192, 0), (4, 6000, 1), (130, 64, 50)])
def test_ln_modulate(rows, hidden, mod):
    P = need_gpu()
    n_mod = -(-rows // mod) if mod else 1
    x, xw = strided(rows, hidden, F32, 12, multiple=4)
    x.copy_(normal((rows, hidden), [rows, hidden], 2.0, 0.5))
    shift, scale = normal((n_mod, hidden), 1, 0.5), normal((n_mod, hidden), 2, 0.5)
    codes, scales = fp8_rows(P, rows, hidden, 20, 1.0)
    P.ln_modulate_fp8(x, shift if mod else shift[0], scale if mod else scale[0], codes, scales, rows_per_mod=mod)
    y = B.ln_modulate(f64(x), f64(shift), f64(scale), mod)
    got, s = B.rows_values(f64(codes), f64(scales)), f64(scales)[:, :rows].T
    # fp32 statistics: sums of `hidden` terms in a tree of 32 / lane and 64 lanes, some ten roundings
    # on the way to y; 64 of them relative to the row's largest parts are ample
    z = np.abs(B.ln_modulate(f64(x), 0 * f64(shift), 0 * f64(scale), mod))
    row = np.arange(rows) // (mod or rows)
    off = 64 * 2.0 ** -24 * ((z + 1) * (1 + np.abs(f64(scale)))[row] + np.abs(f64(shift))[row])
    wide = np.repeat(s, 128, 1)[:, :hidden]
    most = np.stack([np.abs(y[:, g:g + 128]).max(1) for g in range(0, hidden, 128)], 1)
    assert_elementwise(s, most / 448, 0, 64 * 2.0 ** -24 * 8, "scales")
    # a code is off by half a step: 2^-4 of the value, 2^-10 of the scale among the smallest
    assert_elementwise(got, y, (1 + 2.0 ** -4) * off + 1.001 * 2.0 ** -10 * wide, 2.0 ** -4, "values")


def test_nothing_to_do():
    P = need_gpu()
    P.quantize_fp8(torch.zeros(0, 32, device="cuda"), torch.zeros(0, 32, device="cuda").to(E4M3), torch.zeros(1, 0, device="cuda"))
    v = torch.zeros(32, device="cuda")
    P.ln_modulate_fp8(torch.zeros(0, 32, device="cuda"), v, v, torch.zeros(0, 32, device="cuda").to(E4M3), torch.zeros(1, 0, device="cuda"))


def test_refusals():
    P = need_gpu()
    x = torch.zeros(4, 32, device="cuda")
    codes, scales = fp8_rows(P, 4, 32)
    v = torch.zeros(32, device="cuda")
    for args in ((x.half(), codes, scales), (x, codes.float(), scales), (x, codes, scales[:, :3]), (x[0], codes, scales),
                 (x.t(), codes, scales), (x.cpu(), codes, scales), (x, codes.cpu(), scales)):
        with pytest.raises(ValueError):
            P.quantize_fp8(*args)
    with pytest.raises(ValueError, match="rows_per_mod"):
        P.ln_modulate_fp8(x, v, v, codes, scales, rows_per_mod=-1)
    with pytest.raises(ValueError, match="shift"):
        P.ln_modulate_fp8(x, v, v, codes, scales, rows_per_mod=2)
    with pytest.raises(ValueError, match="scale"):
        P.ln_modulate_fp8(x, v, v.bfloat16(), codes, scales)
    with pytest.raises(P.AcidError, match="multiple of 16"):
        P.quantize_fp8(torch.zeros(4, 24, device="cuda"), torch.zeros(4, 24, device="cuda").to(E4M3), scales)
    with pytest.raises(P.AcidError, match="16-byte"):
        P.quantize_fp8(strided(4, 33, F32, 3)[0][:, 1:], codes, scales)
    with pytest.raises(ValueError, match="multiple of 16"):
        P.fp8_shapes(4, 24)
    with pytest.raises(ValueError, match="codes"):
        P.quantize_fp8_weight(x, codes, torch.zeros(1, 1, device="cuda"))
