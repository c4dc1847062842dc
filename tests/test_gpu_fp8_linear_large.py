"""e4m3 products over many tiles a workgroup, in every form that a launch takes: small whole
numbers and scales that are powers of two, so that every output is exact."""
import pytest
import torch

from fp8_form_util import fp8_form
from fp8_util import E4M3
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# rows, outputs, inputs and the form of 8-bit products: more tiles than workgroups, tiles and
# blocks whole and not, one block of inputs, less than one, parts of K
LARGE = [(16640, 1536, 1536, "256x256", 1), (32760, 4608, 1536, "256x256", 1), (33000, 1537, 2064, "256x256", 1),
         (32760, 4601, 1040, "256x256", 1), (33000, 1533, 1536, "128x128", 1), (66000, 1032, 128, "128x128", 1), (60000, 1001, 16, "128x128", 1),
         (20000, 1792, 400, "128x128", 1), (9000, 2301, 656, "128x128", 1), (3000, 4608, 272, "128x128", 1),
         (300, 4608, 8960, "64x64", 1), (1000, 1536, 8960, "64x64", 1), (5000, 200, 144, "64x64", 1),
         (300, 4608, 1536, "64x64", 1), (600, 1001, 8976, "64x64", 3), (64, 1536, 8960, "64x64", 12),
         (1038, 1208, 13824, "128x128", 4), (1038, 1207, 13840, "128x128", 4),
         (633, 1312, 6912, "64x64", 2), (633, 1309, 6928, "64x64", 2), (16, 28672, 1040, "rows", 1), (17, 4608, 1536, "rows", 1), (32, 1001, 8976, "rows", 1), (29, 8176, 400, "rows", 1), (32, 8960, 1536, "64x64", 1), (9, 1001, 8976, "rows", 1), (1, 8960, 1536, "rows", 1)]


@pytest.mark.parametrize("m,n,k,tile,split", LARGE)
@pytest.mark.parametrize("kind,dtype", [("none", BF16), ("none", F32), ("residual", F32)], ids=["bf16", "f32", "residual"])
def test_whole_numbers_are_exact(m, n, k, tile, split, kind, dtype):
    P = need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count == 256:
        assert fp8_form(m, n, k)[:2] == (tile, split)
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    ints = lambda *s: torch.randint(-3, 4, s, generator=g, device="cuda").float()          # noqa: E731
    powers = lambda s: 2.0 ** torch.randint(-1, 2, s, generator=g, device="cuda").float()  # noqa: E731
    a, sa, w, sw = ints(m, k).to(E4M3), powers(P.fp8_shapes(m, k)[1]), ints(n, k).to(E4M3), powers(P.fp8_weight_shapes(n, k)[1])
    bias, gate, residual = ints(n), powers((n,)), ints(m, n)
    out = torch.full((m, n), 77.0, device="cuda", dtype=dtype)
    P.linear_fp8(a, sa, w, sw, out, bias=bias, **(dict(gate=gate, residual=residual) if kind == "residual" else {}))
    av = a.double() * sa[:, :m].t().repeat_interleave(128, 1)[:, :k]
    wv = w.double() * sw.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    y = torch.matmul(av, wv.t().contiguous()) + bias
    if kind == "residual":
        y = residual + gate * y
    assert y.abs().max() < 2 ** 20  # of steps of 1/8: all sums are exact in fp32
    assert torch.equal(out, y.to(dtype))


def test_workspace_of_two_streams_and_forms():
    """Calls that overlap, each with a workspace of its own; and one workspace for calls in turn."""
    P = need_gpu()
    m, n, k = 100, 640, 8960
    assert P.linear_fp8_workspace(m, n, k) > 0
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    ints = lambda *s: torch.randint(-3, 4, s, generator=g, device="cuda").float()  # noqa: E731
    sets = []
    for _ in range(4):
        a, w = ints(m, k).to(E4M3), ints(n, k).to(E4M3)
        one = torch.ones(P.fp8_shapes(m, k)[1], device="cuda"), torch.ones(P.fp8_weight_shapes(n, k)[1], device="cuda")
        sets.append((a, one[0], w, one[1], torch.zeros((m, n), device="cuda"), (a.double() @ w.double().t().contiguous()).float()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, (a, sa, w, sw, out, _) in zip(streams, sets):
            P.linear_fp8(a, sa, w, sw, out, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(out, y) for *_, out, y in sets)
    ws = torch.empty(P.linear_fp8_workspace(m, n, k), dtype=torch.uint8, device="cuda")
    for a, sa, w, sw, out, y in sets:
        out.zero_()
        P.linear_fp8(a, sa, w, sw, out, workspace=ws)
    assert all(torch.equal(out, y) for *_, out, y in sets)
    with pytest.raises(P.AcidError, match="workspace"):
        P.linear_fp8(a, sa, w, sw, out, workspace=ws[:-16])


def test_neighbours_of_the_operands_are_not_used():
    """Rows of a larger matrix on both sides full of NaN, outputs in the middle of a larger one."""
    P = need_gpu()
    for m, n, k in ((5, 100, 144), (40, 100, 400), (1300, 2049, 144), (700, 1536, 640), (16640, 1536, 1536)):
        big = torch.full((m + 64, k + 32), float("nan"), device="cuda").to(E4M3)
        a = big[32:32 + m, 16:16 + k]
        a.copy_(torch.ones((m, k), device="cuda").to(E4M3))
        wide = torch.full((n + 64, k), float("nan"), device="cuda").to(E4M3)
        w = wide[32:32 + n]
        w.copy_(torch.ones((n, k), device="cuda").to(E4M3))
        sa, sw = torch.ones(P.fp8_shapes(m, k)[1], device="cuda"), torch.ones(P.fp8_weight_shapes(n, k)[1], device="cuda")
        for dtype in (BF16, F32):
            whole = torch.full((m + 2, n + 16), -1.0, device="cuda", dtype=dtype)
            out = whole[1:1 + m, 8:8 + n]
            P.linear_fp8(a, sa, w, sw, out)
            assert (out == torch.tensor(float(k), device="cuda").to(dtype)).all(), (m, n, k)
            out.fill_(-1.0)
            assert (whole == -1.0).all()
