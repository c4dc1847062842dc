"""4-bit weights with group scales: conversion bit for bit, products against
64 bits.

Bounds.  Codes and, with fp32 rows in three exact parts, the inputs are exact;
the kernel sums x (16 + c) and takes 24 x away within a group, so with
A = sum_k |x| 40 s (16 + c <= 31, and 24 less 8 + c at most) fp32 accumulation over K
inputs in any order stays below (K / 32 + 200) 2^-24 A: a product of 32 inputs
adds up in one instruction, then blocks, groups and waves.  GELU's slope is
below 1.2; a bf16 output adds half a step.
"""
import numpy as np
import pytest
import torch

from gpu_util import assert_elementwise, need_gpu
from oracle import linear_block as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(t):
    return t.detach().double().cpu().numpy()


def _weights(P, n, k, group, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 31 + n)
    w = 0.02 * torch.randn((k, n), generator=g, device="cuda")
    cs, ss = P.w4_shapes(n, k, group)
    codes = torch.full(cs, 255, dtype=torch.uint8, device="cuda")
    scales = torch.full(ss, 9.0, device="cuda")
    P.quantize_w4(w, codes, scales)
    return w, codes, scales


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(1, 128), (16, 256), (17, 128), (300, 384), (1029, 640)])
def test_quantize_bit_for_bit(group, n, k):
    P = need_gpu()
    w, codes, scales = _weights(P, n, k, group)
    w[:group, 0] = 0.0
    w[0, n // 2] = 1e30
    w[1, n // 3] = 1e-42   # below the smallest normal
    P.quantize_w4(w, codes, scales)
    rc, rs = B.w4_pack(*B.w4_quantize(w.cpu().numpy(), group))
    np.testing.assert_array_equal(scales.cpu().numpy(), rs)
    np.testing.assert_array_equal(codes.cpu().numpy(), rc)


def test_quantize_marks_groups_that_are_not_finite():
    P = need_gpu()
    w, codes, scales = _weights(P, 40, 256, 64)
    w[3, 1], w[70, 2] = float("nan"), float("inf")
    P.quantize_w4(w, codes, scales)
    bad = np.isnan(scales.cpu().numpy())
    assert bad[0, 0, 1] and bad[0, 1, 2] and bad.sum() == 2


def _check(P, m, n, k, group, xt, ot, gelu=False, bias=True, x_pad=0, out_pad=0, seed=0):
    _, codes, scales = _weights(P, n, k, group, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + m)
    x = torch.randn((m, k + x_pad), generator=g, device="cuda").to(DT[xt])[:, :k]
    b = torch.randn(n, generator=g, device="cuda") if bias else None
    wide = torch.full((m, n + out_pad), 7.0, device="cuda").to(DT[ot])
    out = wide[:, :n]
    P.linear_w4(x, codes, scales, out, bias=b, gelu=gelu)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    ref = B.linear_w4(_f64(x), c, s, n, None if b is None else _f64(b), gelu)
    s_n = np.asarray(s, np.float64).transpose(0, 2, 1).reshape(-1, k // group)[:n]
    a = np.abs(_f64(x)) @ (40 * np.repeat(s_n, group, 1)).T
    bound = (k / 32 + 200) * 2.0 ** -24 * a * (1.2 if gelu else 1.0)
    if b is not None:
        bound = bound + 2.0 ** -23 * np.abs(_f64(b))
    if gelu:  # the fast form's exponential and reciprocal: a few steps of y
        y = B.linear_w4(_f64(x), c, s, n, None if b is None else _f64(b))
        bound = bound + 16 * 2.0 ** -24 * (1 + np.abs(y))
    assert_elementwise(_f64(out), ref, bound, 2.0 ** -8 if ot == "bf16" else 2.0 ** -24,
                       f"{m}x{n}x{k} g{group} {xt}->{ot}")
    assert (wide[:, n:] == 7.0).all()


@pytest.mark.parametrize("xt,ot", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("m", [1, 2, 5, 6, 16, 17, 33, 70])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_rows(xt, ot, m, group):
    P = need_gpu()
    _check(P, m, 333, 640, group, xt, ot)


@pytest.mark.parametrize("n,k", [(1, 128), (15, 256), (16, 1024), (49, 1152), (4609, 1536),
                                 (17001, 256), (130, 22016)])
@pytest.mark.parametrize("m", [1, 3, 20])
def test_sizes(n, k, m):
    P = need_gpu()
    _check(P, m, n, k, 128, "bf16", "f32", seed=1)
    _check(P, m, n, k, 32, "f32", "bf16", seed=2)


def test_forms_and_strides():
    P = need_gpu()
    for xt in ("bf16", "f32"):
        for ot in ("bf16", "f32"):
            _check(P, 4, 500, 512, 64, xt, ot, gelu=True)
            _check(P, 4, 500, 512, 64, xt, ot, bias=False, x_pad=24, out_pad=3)
            _check(P, 1, 77, 512, 128, xt, ot, gelu=True, bias=False, x_pad=8, out_pad=5)


def test_rows_and_outputs_keep_to_themselves():
    """A NaN row and a NaN scale touch their own row and output alone."""
    P = need_gpu()
    _, codes, scales = _weights(P, 50, 256, 64)
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn((18, 256), device="cuda").to(dt)
        a, b = (torch.empty((18, 50), device="cuda") for _ in range(2))
        P.linear_w4(x, codes, scales, a)
        x[4, 9] = float("nan")
        s = scales.clone()
        s[1, 2, 5] = float("nan")  # output 21
        P.linear_w4(x, codes, s, b)
        keep = torch.ones_like(a, dtype=torch.bool)
        keep[4] = False
        keep[:, 21] = False
        assert torch.equal(a[keep], b[keep])
        assert b[4].isnan().all() and b[:, 21].isnan().all()


def test_same_bits_on_every_call_stream_and_replay():
    P = need_gpu()
    _, codes, scales = _weights(P, 2000, 2048, 128)
    x = torch.randn((3, 2048), device="cuda").bfloat16()
    want, out = torch.empty(3, 2000, device="cuda"), torch.empty(3, 2000, device="cuda")
    P.linear_w4(x, codes, scales, want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    P.linear_w4(x, codes, scales, out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.linear_w4(x, codes, scales, out)
    for _ in range(3):
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_binding_refuses_on_the_device():
    P = need_gpu()
    _, codes, scales = _weights(P, 50, 256, 64)
    x = torch.zeros((2, 256), device="cuda")
    with pytest.raises(ValueError, match="codes"):
        P.linear_w4(x, codes, scales, torch.zeros((2, 65), device="cuda"))
    with pytest.raises(ValueError, match="bias"):
        P.linear_w4(x, codes, scales, torch.zeros((2, 50), device="cuda"),
                    bias=torch.zeros(49, device="cuda"))
    with pytest.raises(ValueError, match="float16"):
        P.linear_w4(x.half(), codes, scales, torch.zeros((2, 50), device="cuda"))
