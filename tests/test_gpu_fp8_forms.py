"""What acid.h promises of e4m3 products, in every form of them and for every output: NaN stays where it
belongs, padding is not read, scales may be large and small, the same bits each time."""
import pytest
import torch

from fp8_form_util import fp8_form
from fp8_util import E4M3, U16, U32, normal, strided
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# rows (no multiple of 4: scales are padded), outputs, inputs; the form and parts of 8-bit products
FORMS = [(5, 300, 400, "rows", 1), (14, 300, 256, "rows", 1), (30, 300, 1040, "rows", 1), (41, 300, 400, "64x64", 1), (39, 304, 384, "64x64", 1),
         (66, 1536, 8960, "64x64", 8), (601, 1001, 8976, "64x64", 3), (3001, 4608, 256, "128x128", 1), (2998, 4601, 272, "128x128", 1),
         (1038, 1208, 13824, "128x128", 4), (1037, 1207, 13840, "128x128", 4), (16637, 1536, 1536, "256x256", 1), (32757, 4601, 1040, "256x256", 1)]
EACH = pytest.mark.parametrize("m,n,k,tile,split", FORMS, ids=[f"{t}-{m}-{n}-{k}" for m, n, k, t, _ in FORMS])
KINDS = pytest.mark.parametrize("kind", ["bf16", "gelu-bf16", "f32", "gelu-f32", "residual", "residual-exact"])


class Case:
    def __init__(self, m, n, k, tile, split, kind):
        self.P, self.kind = need_gpu(), kind
        if torch.cuda.get_device_properties(0).multi_processor_count == 256:
            assert fp8_form(m, n, k)[:2] == (tile, split)
        self.shape, seed = (m, n), m + n + k
        self.a, self.w = (normal((r, k), [seed, i], 150.0).clamp_(-448, 448).to(E4M3) for i, r in enumerate((m, n)))
        self.sa = normal(self.P.fp8_shapes(m, k)[1], [seed, 2], 0.001, 0.008)
        self.sw = normal(self.P.fp8_weight_shapes(n, k)[1], [seed, 3], 0.001, 0.006) * k ** -0.5
        self.bias, self.gate = normal(n, [seed, 4], 0.1), normal(n, [seed, 5], 0.1, 1.0)
        self.residual = normal((m, n), [seed, 6])

    def run(self, a=None, sa=None, w=None, sw=None, bias=True, **kw):
        out = torch.full(self.shape, 77.0, device="cuda", dtype=BF16 if "bf16" in self.kind else F32)
        if "residual" in self.kind:
            kw.update(gate=self.gate, residual=self.residual if bias else torch.zeros_like(self.residual))
        if "exact" in self.kind:
            kw.update(exact=True)
        self.P.linear_fp8(self.a if a is None else a, self.sa if sa is None else sa, self.w if w is None else w,
                          self.sw if sw is None else sw, out, bias=self.bias if bias else None, gelu="gelu" in self.kind, **kw)
        return out


@EACH
@KINDS
def test_what_is_nan_stays_in_its_row_and_column(m, n, k, tile, split, kind):
    c = Case(m, n, k, tile, split, kind)
    clean = c.run()
    assert torch.isfinite(clean).all()
    a, sa, w, sw = c.a.clone(), c.sa.clone(), c.w.clone(), c.sw.clone()
    a[2, 5] = a[m - 1, k - 1] = w[33, k - 1] = w[n - 1, 0] = float("nan")
    sa[(k - 1) // 128, 1] = sa[0, m - 3] = float("nan")
    sw[1, 0] = float("nan")
    out = c.run(a, sa, w, sw)
    bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    bad[[1, 2, m - 3, m - 1]] = True
    bad[:, 33] = bad[:, n - 1] = True
    bad[:, 128:256] = True
    assert torch.equal(torch.isnan(out), bad)
    assert torch.equal(out[~bad], clean[~bad])


@EACH
@KINDS
def test_padding_is_not_used(m, n, k, tile, split, kind):
    """Scales past the last row, bytes between rows and rows past the last may hold anything."""
    c = Case(m, n, k, tile, split, kind)
    clean = c.run()
    padded, _ = strided(*c.sa.shape, F32, 4, float("nan"), 4)
    padded[:, :m] = c.sa[:, :m]
    wide = torch.full((m + 64, k + 32), float("nan"), device="cuda").to(E4M3)[32:32 + m, 16:16 + k]
    wide.copy_(c.a)
    weight = torch.full((n + 64, k), float("nan"), device="cuda").to(E4M3)[32:32 + n]
    weight.copy_(c.w)
    assert torch.equal(c.run(wide, padded, weight), clean)


@EACH
@pytest.mark.parametrize("kind", ["bf16", "f32", "residual", "residual-exact"])
def test_large_and_small_scales(m, n, k, tile, split, kind):
    """Powers of two in the scales are powers of two in the outputs, bit for bit.  Outputs below 2^-126 (of
    2^-100, some in 2^27 are) have a fixed step there, 2^-133 in bf16 and 2^-149 in fp32: each block's sum
    costs half of fp32's, the output and what it is compared with half of their type's each."""
    c = Case(m, n, k, tile, split, kind)
    plain = c.run(bias=False)
    for x, y in ((60, 40), (-60, -40), (90, -90)):
        out, want = c.run(sa=c.sa * 2.0 ** x, sw=c.sw * 2.0 ** y, bias=False), plain * 2.0 ** (x + y)
        least = want.abs() < 2.0 ** -126
        assert torch.equal(out[~least], want[~least]), (x, y)
        off = (-(-k // 128) + 1) * 2.0 ** -150 + (2.0 ** -133 if kind == "bf16" else 0.0)
        assert ((out[least].double() - want[least].double()).abs() <= off).all(), (x, y)


@EACH
@KINDS
def test_same_bits_with_any_workspace(m, n, k, tile, split, kind):
    c = Case(m, n, k, tile, split, kind)
    first = c.run()
    size = c.P.linear_fp8_workspace(m, n, k)
    assert size or split == 1
    for fill in (255, 0, 127):  # NaN, zeros, large numbers
        ws = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(c.run(workspace=ws), first)


@EACH
@KINDS
def test_against_64_bits(m, n, k, tile, split, kind):
    c = Case(m, n, k, tile, split, kind)
    out = c.run().double()
    av = c.a.double() * c.sa[:, :m].t().double().repeat_interleave(128, 1)[:, :k]
    wv = c.w.double() * c.sw.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    y = torch.matmul(av, wv.t().contiguous()) + c.bias
    # every product, block scale and the bias may cost an fp32 rounding of all that was added; the 8-bit
    # units' cut is 7 2^-13 of the largest of each eight products
    off = (k + 4 * -(-k // 128) + 4) * U32 * (torch.matmul(av.abs(), wv.abs().t().contiguous()) + c.bias.abs())
    if kind in ("bf16", "gelu-bf16", "residual"):
        most = [x.abs().reshape(x.shape[0], -1, 8).amax(2) for x in (av, wv)]
        off += 7 * 2.0 ** -13 * torch.matmul(most[0], most[1].t().contiguous())
    if "gelu" in kind:  # slope below 1.13, and some fp32 roundings of its own
        y = y / 2 * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3)))
        off = 1.13 * off + 16 * U32 * (1 + y.abs())
    if "residual" in kind:
        off = c.gate.abs() * off + 2 * U32 * ((c.gate * y).abs() + c.residual.abs())
        y = c.residual + c.gate * y
    half = U16 if "bf16" in kind else U32
    assert ((out - y).abs() <= (1 + half) * off + half * y.abs()).all()
