"""What the sums of e4m3 products hold: exact products for any output that asks for them, and the
8-bit matrix units' cut, towards zero, within the bound that acid.h states."""
import numpy as np
import pytest
import torch

from fp8_form_util import fp8_form
from fp8_util import E4M3, U16, U32, f64, normal, strided
from gpu_util import assert_elementwise, need_gpu
from oracle import fp8_block as B
from test_gpu_fp8_linear import SIZES, _off, _operands

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
KINDS = pytest.mark.parametrize("kind,dtype", [("none", BF16), ("none", F32), ("gelu", BF16), ("gelu", F32), ("residual", F32)],
                                ids=["bf16", "f32", "gelu-bf16", "gelu-f32", "residual"])


@pytest.mark.parametrize("m,n,k", SIZES)
@KINDS
def test_sizes(m, n, k, kind, dtype):
    """Every output from exact products, within fp32's roundings."""
    P = need_gpu()
    ops, (av, wv) = _operands(P, m, n, k, 20)
    bias, gate, residual = normal(n, 9, 0.3), normal(n, 10), normal((m, n), 11)
    out, whole = strided(m, n, dtype, 3, 5.0)
    P.linear_fp8(*ops, out, bias=bias, gelu=kind == "gelu", exact=True, **(dict(gate=gate, residual=residual) if kind == "residual" else {}))
    off, y = _off(av, wv, f64(bias), True), B.linear(av, wv, f64(bias))
    if kind == "gelu":  # its slope is below 1.13, its own arithmetic good to some fp32 roundings
        y = B.linear(av, wv, f64(bias), gelu=True)
        off = 1.13 * off + 16 * U32 * (1 + np.abs(y))
    elif kind == "residual":
        g, r = f64(gate), f64(residual)
        off = np.abs(g) * off + 2 * U32 * (np.abs(g * y) + np.abs(r))
        y = r + g * y
    assert_elementwise(f64(out), y, (1 + U16) * off + 2.0 ** -133, U16 if dtype == BF16 else U32, f"{kind} {m} x {n} x {k}")
    assert (whole[:, n:] == 5.0).all()
    if dtype == F32 and kind != "residual":  # what these outputs come from in any case
        plain = torch.zeros((m, n), device="cuda")
        P.linear_fp8(*ops, plain, bias=bias, gelu=kind == "gelu")
        assert torch.equal(plain, out)


# rows, outputs, inputs and the form of exact products: tiles and blocks whole and not, parts of K
LARGE = [(16640, 1536, 1536, "128x128", 1), (33000, 1537, 2064, "128x128", 1), (20000, 1792, 400, "128x128", 1), (5000, 200, 144, "64x64", 1),
         (300, 1001, 1040, "64x64", 1), (600, 1001, 8976, "128x128", 8), (64, 1536, 8960, "64x64", 12), (1038, 1208, 13824, "128x128", 6),
         (1038, 1207, 13840, "128x128", 6), (32, 1001, 8976, "rows", 1), (9, 1001, 8976, "rows", 1), (1, 8960, 1536, "rows", 1)]


@pytest.mark.parametrize("m,n,k,tile,split", LARGE)
@pytest.mark.parametrize("kind,dtype", [("none", BF16), ("residual", F32)], ids=["bf16", "residual"])
def test_whole_numbers(m, n, k, tile, split, kind, dtype):
    """Small whole numbers and scales that are powers of two, over many tiles: exact in fp32."""
    P = need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert fp8_form(m, n, k, True)[:2] == (tile, split)
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    ints = lambda *s: torch.randint(-3, 4, s, generator=g, device="cuda").float()          # noqa: E731
    powers = lambda s: 2.0 ** torch.randint(-1, 2, s, generator=g, device="cuda").float()  # noqa: E731
    a, sa, w, sw = ints(m, k).to(E4M3), powers(P.fp8_shapes(m, k)[1]), ints(n, k).to(E4M3), powers(P.fp8_weight_shapes(n, k)[1])
    bias, gate, residual = ints(n), powers((n,)), ints(m, n)
    out = torch.full((m, n), 77.0, device="cuda", dtype=dtype)
    P.linear_fp8(a, sa, w, sw, out, bias=bias, exact=True, **(dict(gate=gate, residual=residual) if kind == "residual" else {}))
    av = a.double() * sa[:, :m].t().repeat_interleave(128, 1)[:, :k]
    wv = w.double() * sw.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    y = torch.matmul(av, wv.t().contiguous()) + bias
    if kind == "residual":
        y = residual + gate * y
    assert y.abs().max() < 2 ** 20  # of steps of 1/8: all sums are exact in fp32
    assert torch.equal(out, y.to(dtype))


# a size for each form of 8-bit products
FORMS = [(4, 200, 400, "rows"), (30, 200, 256, "rows"), (40, 260, 400, "64x64"), (64, 1536, 8960, "64x64"), (3001, 4608, 256, "128x128"),
         (3000, 4601, 272, "128x128"), (1038, 1208, 13824, "128x128"), (16637, 1536, 1536, "256x256"), (32760, 4601, 1040, "256x256")]
EACH_FORM = pytest.mark.parametrize("m,n,k,tile", FORMS)


def _form(m, n, k, tile):
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert fp8_form(m, n, k)[0] == tile


def _ones(P, m, n, k):
    return torch.ones(P.fp8_shapes(m, k)[1], device="cuda"), torch.ones(P.fp8_weight_shapes(n, k)[1], device="cuda")


def _cut(a, w):
    """7 2^-13 of the largest of each eight products."""
    most = [x.double().abs().reshape(x.shape[0], -1, 8).amax(2) for x in (a, w)]
    return 7 * 2.0 ** -13 * torch.matmul(most[0], most[1].t().contiguous())


@EACH_FORM
@pytest.mark.parametrize("kind,dtype", [("none", BF16), ("residual", F32)], ids=["bf16", "residual"])
def test_beside_outliers(m, n, k, tile, kind, dtype):
    """Small whole numbers beside one large product, and beside two that cancel, among the same eight:
    exact products keep them all (sums below 2^24), the 8-bit units leave them within the cut."""
    P = need_gpu()
    _form(m, n, k, tile)
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    a, w = (torch.randint(-3, 4, s, generator=g, device="cuda").float() for s in ((m, k), (n, k)))
    a[:, 8], w[:, 8] = 448, 448
    a[:, 13], w[:, 13] = -448, 448
    a[:, k - 1], w[:, k - 1] = 448, -448
    a, w = a.to(E4M3), w.to(E4M3)
    sa, sw = _ones(P, m, n, k)
    gate, residual = torch.ones(n, device="cuda"), torch.randint(-3, 4, (m, n), generator=g, device="cuda").float()
    kw = dict(gate=gate, residual=residual) if kind == "residual" else {}
    y = torch.matmul(a.double(), w.double().t().contiguous())
    if kind == "residual":
        y = y + residual
    assert y.abs().max() < 2 ** 23
    out = torch.full((m, n), 77.0, device="cuda", dtype=dtype)
    P.linear_fp8(a, sa, w, sw, out, exact=True, **kw)
    assert torch.equal(out, y.to(dtype))
    out.fill_(77.0)
    P.linear_fp8(a, sa, w, sw, out, **kw)
    # the cut, the blocks' sums in fp32 (below 2^19) and the output's rounding
    off = _cut(a, w) + (k / 128 + 2) * U32 * 2.0 ** 19
    half = U16 if dtype == BF16 else U32
    assert ((out.double() - y).abs() <= (1 + half) * off + half * y.abs()).all()


@EACH_FORM
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "residual"])
def test_the_cut_has_no_side(m, n, k, tile, dtype):
    """Rows of the other sign give sums of the other sign, bit for bit: what is dropped has no side.
    Operands of one sign lose: their sums are not above the exact ones by more than fp32's roundings."""
    P = need_gpu()
    _form(m, n, k, tile)
    a, w = (normal(s, [m, i], 150.0).clamp_(-448, 448) for i, s in enumerate(((m, k), (n, k))))
    sa, sw = _ones(P, m, n, k)
    kw = dict(gate=torch.ones(n, device="cuda"), residual=torch.zeros((m, n), device="cuda")) if dtype == F32 else {}
    outs = []
    for rows in (a, -a, a.abs()):
        out = torch.full((m, n), 77.0, device="cuda", dtype=dtype)
        P.linear_fp8(rows.to(E4M3), sa, (w.abs() if rows.min() >= 0 else w).to(E4M3), sw, out, **kw)
        outs.append(out)
    assert torch.equal(outs[0], -outs[1])
    pa, pw = a.abs().to(E4M3), w.abs().to(E4M3)
    y = torch.matmul(pa.double(), pw.double().t().contiguous())
    half = U16 if dtype == BF16 else U32
    got, roundings = outs[2].double(), (k / 8 + k / 128 + 4) * U32 * y  # a sum of eights, and of blocks
    assert (got <= y + roundings + half * y).all()
    assert (got >= y - _cut(pa, pw) - roundings - half * y).all()
