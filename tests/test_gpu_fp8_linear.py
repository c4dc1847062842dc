"""e4m3 products with block scales against the same products in 64 bits."""
import numpy as np
import pytest
import torch

from fp8_util import E4M3, U16, U32, f64, fp8_rows, normal, quantized_rows, quantized_weight, strided
from gpu_util import assert_elementwise, need_gpu
from oracle import fp8_block as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# (rows, outputs, inputs): a token, a few, tiles whole and not, blocks whole and not, long
# rows of few outputs
SIZES = [(1, 1, 16), (1, 16, 16), (1, 129, 144), (2, 128, 128), (3, 1000, 8960), (7, 2048, 1536), (15, 100, 2064), (16, 257, 1040), (17, 100, 272),
         (31, 96, 4096), (32, 640, 256), (33, 65, 128), (48, 1536, 2048), (63, 64, 656), (64, 128, 384), (65, 300, 8192), (100, 48, 8960), (127, 129, 400),
         (128, 128, 128), (129, 384, 1040), (200, 1000, 528), (256, 256, 768), (257, 513, 528), (300, 1001, 1040),
         (512, 512, 1024), (511, 256, 2048), (700, 1536, 640), (1000, 300, 2064), (1300, 2049, 144), (2000, 1024, 272)]


def _operands(P, m, n, k, seed=0):
    """e4m3 operands (rows strided), as tensors, and their values in 64 bits."""
    a, a_scales = fp8_rows(P, m, k, 16)
    P.quantize_fp8(normal((m, k), [seed, m, k], 1.0, 0.2), a, a_scales)
    w, w_scales = quantized_weight(P, normal((k, n), [seed + 1, n, k], k ** -0.5, 0.1 * k ** -0.5))
    return (a, a_scales, w, w_scales), (B.rows_values(f64(a), f64(a_scales)), B.weight_values(f64(w), f64(w_scales)))


def _off(av, wv, bias, exact):
    """Bound of the sums.  Exact products: every one of the K, block scales and the bias may
    cost an fp32 rounding of all that was added.  The 8-bit matrix units also cut, in each
    eight neighbouring products, what lies below 2^-13 of the largest: seven times that."""
    k = av.shape[1]
    off = (k + 4 * -(-k // 128) + 4) * U32 * (np.abs(av) @ np.abs(wv).T + np.abs(bias))
    if not exact:
        most = [np.abs(x).reshape(x.shape[0], -1, 8).max(2) for x in (av, wv)]
        off = off + 7 * 2.0 ** -13 * (most[0] @ most[1].T)
    return off


def _check(out, av, wv, bias, kind="none", gate=None, residual=None, what=""):
    off = _off(av, wv, bias, out.dtype == F32 and kind != "residual")
    y = B.linear(av, wv, bias)
    if kind == "gelu":  # its slope is below 1.13, its own arithmetic good to some fp32 roundings
        y = B.linear(av, wv, bias, gelu=True)
        off = 1.13 * off + 16 * U32 * (1 + np.abs(y))
    elif kind == "residual":
        off = np.abs(gate) * off + 2 * U32 * (np.abs(gate * y) + np.abs(residual))
        y = residual + gate * y
    rtol = U16 if out.dtype == BF16 else U32
    assert_elementwise(f64(out), y, (1 + U16) * off + 2.0 ** -133, rtol, what)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind,dtype", [("none", BF16), ("none", F32), ("residual", F32)], ids=["bf16", "f32", "residual"])
def test_whole_numbers_are_exact(m, n, k, kind, dtype):
    """Small whole numbers and scales that are powers of two: every sum is exact in fp32 (and
    no product lies far below another), so the outputs are the oracle's, rounded once."""
    P = need_gpu()
    rng = np.random.default_rng([m, n, k])
    ints = lambda *s: torch.from_numpy(rng.integers(-3, 4, s).astype(np.float32)).cuda()  # noqa: E731
    powers = lambda s: torch.from_numpy(2.0 ** rng.integers(-1, 2, s)).float().cuda()     # noqa: E731
    a, sa, w, sw = ints(m, k).to(E4M3), powers(P.fp8_shapes(m, k)[1]), ints(n, k).to(E4M3), powers(P.fp8_weight_shapes(n, k)[1])
    bias, gate, residual = ints(n), powers(n), ints(m, n)
    out = torch.zeros((m, n), device="cuda", dtype=dtype)
    P.linear_fp8(a, sa, w, sw, out, bias=bias, **(dict(gate=gate, residual=residual) if kind == "residual" else {}))
    y = B.linear(B.rows_values(f64(a), f64(sa)), B.weight_values(f64(w), f64(sw)), f64(bias),
                 **(dict(gate=f64(gate), residual=f64(residual)) if kind == "residual" else {}))
    assert np.abs(y).max() < 2.0 ** 18  # of steps of 1/8
    assert torch.equal(out.cpu(), torch.from_numpy(y).to(dtype))


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("kind,dtype", [("none", BF16), ("none", F32), ("gelu", BF16), ("gelu", F32), ("residual", F32)],
                         ids=["bf16", "f32", "gelu-bf16", "gelu-f32", "residual"])
def test_sizes(m, n, k, kind, dtype):
    P = need_gpu()
    ops, (av, wv) = _operands(P, m, n, k)
    bias = normal(n, 9, 0.3)
    out, whole = strided(m, n, dtype, 3, 5.0)
    gate = normal(n, 10) if kind == "residual" else None
    residual = None
    if kind == "residual":
        residual, _ = strided(m, n, F32, 1)
        residual.copy_(normal((m, n), 11))
    P.linear_fp8(*ops, out, bias=bias, gelu=kind == "gelu", gate=gate, residual=residual)
    _check(out, av, wv, f64(bias), kind, *(() if gate is None else (f64(gate), f64(residual))), what=f"{kind} {m} x {n} x {k}")
    assert (whole[:, n:] == 5.0).all()


@pytest.mark.parametrize("m,n,k", [(1, 300, 1040), (20, 256, 512), (256, 256, 512), (300, 300, 400)])
def test_without_bias_and_in_place(m, n, k):
    P = need_gpu()
    ops, (av, wv) = _operands(P, m, n, k, 5)
    out = torch.empty((m, n), device="cuda")
    P.linear_fp8(*ops, out)
    _check(out, av, wv, np.zeros(n))
    gate, h = normal(n, 1), normal((m, n), 2)
    before = f64(h)
    P.linear_fp8(*ops, h, gate=gate, residual=h)
    _check(h, av, wv, np.zeros(n), "residual", f64(gate), before)


@pytest.mark.parametrize("m,n,k", [(4, 200, 400), (40, 200, 400), (300, 260, 400), (600, 512, 1024)])
def test_what_is_nan_stays_in_its_row_and_column(m, n, k):
    P = need_gpu()
    (a, sa, w, sw), (av, wv) = _operands(P, m, n, k, 7)
    a[2, 5] = float("nan")
    w[33, k - 1] = float("nan")
    sa[(k - 1) // 128, 1] = float("nan")
    sw[1, 0] = float("nan")
    out = torch.empty((m, n), device="cuda")
    P.linear_fp8(a, sa, w, sw, out)
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[1:3] = True
    bad[:, 33] = True
    bad[:, 128:256] = True
    assert torch.equal(torch.isnan(out), bad)
    keep = ~bad.cpu().numpy()
    off = _off(av, wv, 0.0, True)
    assert_elementwise(f64(out)[keep], B.linear(av, wv)[keep], off[keep], U32)


@pytest.mark.parametrize("m", [1, 5, 16, 30, 64, 130, 300, 520])
def test_padding_of_scales_is_not_used(m):
    """Scales past the last row, and rows past the strides' width, may hold anything."""
    P = need_gpu()
    n, k = 260, 400
    (a, sa, w, sw), (av, wv) = _operands(P, m, n, k, 8)
    padded, _ = strided(*sa.shape, F32, 4, float("nan"), 4)
    padded[:, :m] = sa[:, :m]
    wide, whole = strided(m, k, E4M3, 32, float("nan"), 16)
    wide.copy_(a)
    out = torch.empty((m, n), device="cuda")
    P.linear_fp8(wide, padded, w, sw, out)
    _check(out, av, wv, np.zeros(n))


def test_large_and_small_scales():
    """Scales whose products leave the ordinary range: the sums go with them."""
    P = need_gpu()
    m, n, k = 40, 130, 256
    (a, sa, w, sw), _ = _operands(P, m, n, k, 12)
    for x, y in ((2.0 ** 60, 2.0 ** 40), (2.0 ** -60, 2.0 ** -40), (2.0 ** 90, 2.0 ** -90)):
        sa2, sw2 = sa * x, sw * y
        out = torch.empty((m, n), device="cuda")
        P.linear_fp8(a, sa2, w, sw2, out)
        _check(out, B.rows_values(f64(a), f64(sa2)), B.weight_values(f64(w), f64(sw2)), np.zeros(n))


@pytest.mark.parametrize("m,n,k", [(1, 1536, 8960), (8, 1536, 8960), (64, 512, 4096), (256, 1536, 8960), (600, 700, 2048)])
def test_same_bits_each_time_and_with_a_callers_workspace(m, n, k):
    P = need_gpu()
    ops, _ = _operands(P, m, n, k, 3)
    first = torch.empty((m, n), device="cuda")
    P.linear_fp8(*ops, first)
    ws = torch.full((P.linear_fp8_workspace(m, n, k),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        out = torch.full((m, n), 9.0, device="cuda")
        P.linear_fp8(*ops, out, workspace=ws)
        assert torch.equal(out, first)


def test_codes_of_every_value():
    """All 254 finite codes as rows against unit weights: products are exact."""
    P = need_gpu()
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)[:, None].repeat(1, 16).cuda()
    codes[127], codes[255] = 0, 0
    a = torch.zeros((256, 16), dtype=torch.uint8, device="cuda")
    a[:, 3] = codes[:, 0]
    a = a.view(E4M3)
    sa = torch.ones((1, 256), device="cuda")
    w = torch.zeros((32, 16), device="cuda")
    w[torch.arange(32), 3] = 2.0 ** (torch.arange(32, device="cuda") % 12 - 4.0)
    w, sw = w.to(E4M3), torch.full((1, 1), 0.5, device="cuda")
    for rows in (256, 12):
        out = torch.empty((rows, 32), device="cuda")
        P.linear_fp8(a[:rows], sa[:, :rows], w, sw, out)
        assert torch.equal(out, a[:rows, 3:4].float() * (0.5 * w[:, 3].float())[None])


def test_offsets_past_32_bits():
    """Rows far apart, and an output of more than 2^31 elements' reach."""
    P = need_gpu()
    m, n, k, ld = 300, 256, 256, (1 << 23) + 64  # 2.5 GB of rows; outputs 10 GB apart
    (a, sa, w, sw), (av, wv) = _operands(P, m, n, k, 4)
    far = torch.zeros((m, ld), dtype=torch.uint8, device="cuda").view(E4M3)[:, :k]
    far.copy_(a)
    out = torch.zeros((m, ld), device="cuda")[:, :n]
    P.linear_fp8(far, sa, w, sw, out)
    _check(out, av, wv, np.zeros(n))
    out.zero_()
    P.linear_fp8(far[:3], sa[:, :4], w, sw, out[:3])
    _check(out[:3], av[:3], wv, np.zeros(n))
    assert not out[3:].any()


def test_refusals():
    P = need_gpu()
    (a, sa, w, sw), _ = _operands(P, 5, 40, 64)
    out, v = torch.zeros((5, 40), device="cuda"), torch.zeros(40, device="cuda")
    P.linear_fp8(a[:0], sa[:, :0], w, sw, out[:0])
    for args, kw in (((a.float(), sa, w, sw, out), {}), ((a, sa[:, :5], w, sw, out), {}), ((a, sa, w[:39], sw, out), {}),
                     ((a, sa, w, sw[:0], out), {}), ((a, sa, w, sw, out.half()), {}), ((a, sa, w, sw, out), dict(bias=v[:3])),
                     ((a, sa, w, sw, out), dict(gate=v)), ((a, sa, w, sw, out), dict(residual=out)),
                     ((a, sa, w, sw, out), dict(gate=v, residual=out, gelu=True)), ((a, sa, w.cpu(), sw, out), {}),
                     ((a[0], sa, w, sw, out), {}), ((a, sa, w, sw, out.t()), {})):
        with pytest.raises(ValueError):
            P.linear_fp8(*args, **kw)
    with pytest.raises(P.AcidError, match="fp32"):
        P.linear_fp8(a, sa, w, sw, out.bfloat16(), gate=v, residual=out)
    with pytest.raises(P.AcidError, match="overlaps"):
        P.linear_fp8(a, sa, w, sw, out, bias=out[0])
