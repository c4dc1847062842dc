"""The seam between two blocks against its definition in 64 bits.

Bounds.  A row's statistics are sums of at most 8192 values over a tree of
threads: fewer than 64 + 16 + 10 roundings deep, so relative errors below
100 x 2^-24 of the sums of absolute values.  With n = (x - mean) r, an error dx
of x and the statistics' own give |dn| <= r (dx + mean(dx)) + |n| (r mean(|n| dx)
+ 100 x 2^-24) + 100 x 2^-24 r mean|x| + 4 x 2^-24 |n|, which is carried from y
to h' to out; a bf16 output adds half a step.
"""
import numpy as np
import pytest
import torch

from gpu_util import assert_elementwise, need_gpu
from oracle import linear_block as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def _f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def _norm_error(x, dx, kind, eps):
    if kind == "none":
        return dx
    c = x - x.mean(1, keepdims=True) if kind == "layer" else x
    r = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    n, m = c * r, lambda z: z.mean(1, keepdims=True)
    return (r * (dx + m(dx)) + np.abs(n) * (r * m(np.abs(n) * dx) + 104 * U)
            + 100 * U * r * m(np.abs(x)))


class Seam:
    def __init__(self, rows, hidden, y="bf16", out="bf16", post="rms", pre="layer", weights=True,
                 mods=0, gate=True, modulate=True, pad=0, seed=0, res_scale=0.9, eps=1e-6):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed * 977 + hidden)

        def rnd(*s, m=0.0):
            return torch.randn(s, generator=g, device="cuda") + m

        def wide(t):  # a row-strided view
            w = torch.full((t.shape[0], t.shape[1] + pad), 7.0, device="cuda").to(t.dtype)
            w[:, :t.shape[1]] = t
            return w[:, :t.shape[1]]

        n_mod = -(-rows // mods) if mods else 1
        self.h = wide(2 * rnd(rows, hidden, m=0.4))
        self.y = None if y is None else wide((3 * rnd(rows, hidden, m=-0.5)).to(DT[y]))
        self.out = None if out is None else wide(torch.full((rows, hidden), 7.0, device="cuda").to(DT[out]))
        self.h_out = None if y is None else wide(torch.full((rows, hidden), 7.0, device="cuda"))
        self.kw = dict(res_scale=res_scale, post=post, pre=pre, rows_per_mod=mods, eps=eps,
                       post_weight=rnd(hidden, m=1) if weights else None,
                       pre_weight=rnd(hidden, m=1) if weights else None,
                       gate=rnd(n_mod, hidden) if gate else None,
                       shift=rnd(n_mod, hidden) if modulate else None,
                       scale=rnd(n_mod, hidden) if modulate else None)

    def run(self, P, **kw):
        P.residual_norm(self.h, self.y, h_out=self.h_out, out=self.out, **self.kw, **kw)
        return self

    def check(self, what=""):
        kw = {k: _f64(v) if torch.is_tensor(v) else v for k, v in self.kw.items()}
        h, y = _f64(self.h), _f64(self.y)
        h1, out = B.residual_norm(h, y, **kw)
        rows = h.shape[0]
        at = np.arange(rows) // (kw["rows_per_mod"] or rows)
        vec = lambda name, d: d if kw[name] is None else np.abs(kw[name])[at]  # noqa: E731
        dh = np.zeros_like(h)
        if y is not None:
            pw = 1.0 if kw["post_weight"] is None else np.abs(kw["post_weight"])
            dy = _norm_error(y, np.zeros_like(y), kw["post"], kw["eps"])
            ny = np.abs(B.norm(y, kw["post"], kw["eps"])) * pw * vec("gate", 1.0)
            dh = dy * pw * vec("gate", 1.0) + 4 * U * ny + 2 * U * (np.abs(h) * abs(kw["res_scale"]) + ny)
            assert_elementwise(_f64(self.h_out), h1, dh, 0.0, f"{what} h")
        if self.out is not None:
            w = 1.0 if kw["pre_weight"] is None else np.abs(kw["pre_weight"])
            dn = _norm_error(h1, dh, kw["pre"], kw["eps"])
            s = 1.0 if kw["scale"] is None else np.abs(1 + kw["scale"])[at] + 2 * U
            n = np.abs(B.norm(h1, kw["pre"], kw["eps"])) * w
            d = (dn * w + 4 * U * n) * s + 4 * U * (n * s + vec("shift", 0.0))
            assert_elementwise(_f64(self.out), out, 1.01 * d,
                               2.0 ** -8 if self.out.dtype == torch.bfloat16 else U, f"{what} out")
        for t in (self.h, self.y, self.out, self.h_out):  # between the rows
            if t is not None and t.stride(0) > t.shape[1]:
                whole = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))
                assert (whole[:, t.shape[1]:] == 7.0).all()


@pytest.mark.parametrize("hidden", [4, 8, 64, 252, 256, 260, 512, 516, 1024, 1028, 1536, 1540, 2048,
                                    2052, 4096, 4100, 6148, 8188, 8192])
@pytest.mark.parametrize("rows", [1, 3, 9])
def test_widths(hidden, rows):
    P = need_gpu()
    for k, (y, out) in enumerate((("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"))):
        Seam(rows, hidden, y, out, seed=k).run(P).check(f"{rows}x{hidden} {y}->{out}")


@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("weights,gate,modulate", [(True, True, True), (False, False, False),
                                                   (True, False, True), (False, True, False)])
def test_forms(post, pre, weights, gate, modulate):
    P = need_gpu()
    for rows, hidden in ((5, 320), (2, 4352), (700, 1536)):
        Seam(rows, hidden, "f32", "f32", post, pre, weights, 0, gate, modulate).run(P).check()


@pytest.mark.parametrize("rows,mods", [(1, 1), (7, 1), (7, 2), (7, 7), (7, 100), (1000, 250),
                                       (1001, 333), (4099, 13)])
@pytest.mark.parametrize("hidden", [256, 4608])
def test_modulation_rows(rows, mods, hidden):
    P = need_gpu()
    Seam(rows, hidden, "bf16", "bf16", mods=mods, seed=mods).run(P).check(f"mods {mods}")


@pytest.mark.parametrize("hidden", [128, 1536, 4224])
def test_row_strides(hidden):
    P = need_gpu()
    Seam(37, hidden, "bf16", "bf16", pad=12).run(P).check("strided")
    Seam(37, hidden, "f32", "f32", pad=4, mods=10).run(P).check("strided")


@pytest.mark.parametrize("rows,hidden", [(1, 1536), (900, 1536), (3, 6000)])
def test_in_place_and_parts(rows, hidden):
    P = need_gpu()
    s = Seam(rows, hidden).run(P)
    h = s.h.clone()
    P.residual_norm(h, s.y, **dict(s.kw))                        # no out, in place
    assert torch.equal(h, s.h_out)
    out = torch.empty_like(s.out)
    P.residual_norm(h, None, out=out, **dict(s.kw))              # then out alone
    assert torch.equal(out, s.out)
    h = s.h.clone()
    out.zero_()
    P.residual_norm(h, s.y, out=out, **s.kw)                     # both, in place
    assert torch.equal(h, s.h_out) and torch.equal(out, s.out)


def test_rows_keep_to_themselves():
    """A row of NaN, of infinities, of zeros, and a constant one: the others
    are as they were without them."""
    P = need_gpu()
    for hidden in (256, 4352):
        s = Seam(12, hidden, "f32", "f32").run(P)
        h, out = s.h_out.clone(), s.out.clone()
        s.y[3], s.h[5], s.y[7], s.h[7] = float("nan"), float("inf"), 0.0, 0.0
        s.y[9] = 2.5
        s.run(P)
        keep = [0, 1, 2, 4, 6, 8, 10, 11]
        assert torch.equal(s.h_out[keep], h[keep]) and torch.equal(s.out[keep], out[keep])
        assert s.h_out[3].isnan().all() and s.out[5].isnan().all()
        assert (s.h_out[7] == 0).all() and torch.isfinite(s.out[[7, 9]]).all()


def test_large_mean_keeps_its_variance():
    """Rows at 1000 with a spread of 1: the centred pass keeps LayerNorm exact."""
    P = need_gpu()
    s = Seam(6, 1536, "f32", "f32", post="layer", pre="layer")
    s.y += 1000.0
    s.h += 1000.0
    s.run(P).check("large mean")


def test_captured_and_on_another_stream():
    P = need_gpu()
    s = Seam(300, 1536, mods=77).run(P)
    h, out = s.h_out.clone(), s.out.clone()
    side = torch.cuda.Stream()
    s.out.zero_()
    torch.cuda.synchronize()
    s.run(P, stream=side)
    side.synchronize()
    assert torch.equal(s.out, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run(P)
    for _ in range(3):
        s.h_out.zero_()
        s.out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.h_out, h) and torch.equal(s.out, out)


def test_binding_refuses_on_the_device():
    P = need_gpu()
    h = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError, match="gate"):
        P.residual_norm(h, h.clone(), gate=torch.zeros(2, 64, device="cuda"))
    with pytest.raises(ValueError, match="unit column stride"):
        P.residual_norm(h, torch.zeros(64, 4, device="cuda").t())
    with pytest.raises(P.AcidError, match="overlaps"):
        P.residual_norm(h, h.clone(), out=h)
    assert (h == 0).all()
