"""The 8-bit block's operators as they are used together: a DiT block on its
residual stream, eager, captured into graphs and on several streams."""
import numpy as np
import pytest
import torch

from fp8_util import E4M3, U16, U32, f64, normal, quantized_weight
from gpu_util import assert_elementwise, attention_bound, need_gpu, rel_err
from oracle import fp8_block as B
import oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
HEADS, D, H, FFN = 4, 64, 256, 1040   # an MLP width that is no whole blocks
SECTIONS = (12, 10, 10)


class Block:
    """Weights, buffers and the calls of one block over `tokens` tokens (text first)."""

    def __init__(self, P, tokens, text, seed=0):
        self.P, self.L = P, tokens
        w = lambda i, k, n: normal((k, n), [seed, i], k ** -0.5)  # noqa: E731
        self.full = [w(1, H, 3 * H), w(2, H, H), w(3, H, FFN), w(4, FFN, H)]
        self.w = [quantized_weight(P, x) for x in self.full]
        self.b = [normal(n, [seed, 10 + n], 0.1) for n in (3 * H, H, FFN, H - 1 + 1)]
        self.mod = [normal(H, [seed, 20 + i], 0.3) for i in range(6)]
        self.q_weight, self.k_weight = normal(H, [seed, 30], 0.1, 1.0), normal(H, [seed, 31], 0.1, 1.0)
        side = 4
        at = torch.arange(tokens - text)
        self.pos = torch.zeros((3, tokens), dtype=torch.int32)
        self.pos[:, text:] = torch.stack((at // (side * side), at // side % side, at % side))
        self.pos = self.pos.cuda()
        self.freqs = torch.cat([100.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in SECTIONS]).cuda()
        e = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        rows = lambda k: (e(*P.fp8_shapes(tokens, k)[0], dtype=E4M3), e(*P.fp8_shapes(tokens, k)[1], dtype=F32))  # noqa: E731
        self.x8, self.o8, self.y8, self.u8 = rows(H), rows(H), rows(H), rows(FFN)
        self.qkv, self.o, self.u = e(tokens, 3 * H), e(tokens, H), e(tokens, FFN)
        self.q, self.k = e(HEADS, tokens, D), e(HEADS, tokens, D)
        self.vt = e(HEADS, D, (tokens + 7) // 8 * 8)
        self.h = e(tokens, H, dtype=F32)

    def run(self, stream=None, workspace=None):
        P, (sh1, sc1, g1, sh2, sc2, g2) = self.P, self.mod
        kw = dict(stream=stream)
        ws = dict(stream=stream, workspace=workspace)
        P.ln_modulate_fp8(self.h, sh1, sc1, *self.x8, **kw)
        P.linear_fp8(*self.x8, *self.w[0], self.qkv, bias=self.b[0], **ws)
        P.rotary_qkv(self.qkv[:, :H], self.qkv[:, H:2 * H], self.qkv[:, 2 * H:], self.pos, self.freqs, SECTIONS, self.q, self.k,
                     self.vt[:, :, :self.L], norm="rms_row", q_weight=self.q_weight, k_weight=self.k_weight, q_scale=P.q_scale(D), **kw)
        P.attention(self.q, self.k, self.vt, self.o, q_prescaled=True, **kw)
        P.quantize_fp8(self.o, *self.o8, **kw)
        P.linear_fp8(*self.o8, *self.w[1], self.h, bias=self.b[1], gate=g1, residual=self.h, **ws)
        P.ln_modulate_fp8(self.h, sh2, sc2, *self.y8, **kw)
        P.linear_fp8(*self.y8, *self.w[2], self.u, bias=self.b[2], gelu=True, **ws)
        P.quantize_fp8(self.u, *self.u8, **kw)
        P.linear_fp8(*self.u8, *self.w[3], self.h, bias=self.b[3], gate=g2, residual=self.h, **ws)

    def state(self):
        return [t.clone() for t in (self.h, self.qkv, self.q, self.k, self.vt, self.o, self.u, *self.x8, *self.u8)]

    def workspace(self):
        return max(self.P.linear_fp8_workspace(self.L, n, k) for n, k in ((3 * H, H), (H, H), (FFN, H), (H, FFN)))


def _same(a, b):
    return all(torch.equal(x.float(), y.float()) for x, y in zip(a, b))


@pytest.mark.parametrize("tokens,text", [(1, 0), (70, 6), (300, 44)])
def test_block(tokens, text):
    P = need_gpu()
    b = Block(P, tokens, text)
    h0 = normal((tokens, H), 5)
    b.h.copy_(h0)
    b.run()
    W = [B.weight_values(f64(c), f64(s)) for c, s in b.w]
    bias, mod = [f64(x) for x in b.b], [f64(x) for x in b.mod]

    def product(rows, i, **kw):
        return B.linear(B.rows_values(f64(rows[0]), f64(rows[1])), W[i], bias[i], **kw)

    # each step from what the one before left, within what its own roundings allow
    x = B.rows_values(f64(b.x8[0]), f64(b.x8[1]))
    ref = B.ln_modulate(f64(h0), mod[0], mod[1])
    assert_elementwise(x, ref, 2.0 ** -10 * np.abs(ref).max(1, keepdims=True) / 448 * 1.01 + 1e-5, 2.0 ** -4 * 1.01, "x")
    assert_elementwise(f64(b.qkv), product(b.x8, 0), 2.0 ** -8 * np.abs(x).max(), U16, "qkv")
    qkv = f64(b.qkv)
    for got, at, w, s in ((b.q, 0, b.q_weight, P.q_scale(D)), (b.k, 1, b.k_weight, 1.0)):
        want = B.heads(qkv[:, at * H:(at + 1) * H], HEADS, f64(b.pos), f64(b.freqs), SECTIONS, norm="rms_row", weight=f64(w), scale=s)
        assert_elementwise(f64(got), want, 64 * U32 * np.abs(want).max(), U16, "heads")
    assert torch.equal(b.vt[:, :, :tokens], b.qkv[:, 2 * H:].reshape(tokens, HEADS, D).permute(1, 2, 0))
    # attention's own tests bound it; here: it was given what it takes
    plain_q, k, v = f64(b.q) / P.q_scale(D), f64(b.k), f64(b.vt[:, :, :tokens]).transpose(0, 2, 1)
    o, atol = (np.concatenate([f(plain_q[i], k[i], v[i]) for i in range(HEADS)], 1) for f in (O.attention, attention_bound))
    assert_elementwise(f64(b.o), o, atol, U16, "attention")
    codes, scales = B.quantize_rows(b.u.float().cpu().numpy())
    assert np.array_equal(f64(b.u8[0]), codes) and np.array_equal(f64(b.u8[1])[:, :tokens], scales.astype(np.float64))
    assert_elementwise(f64(b.u), product(b.y8, 2, gelu=True), 2.0 ** -8, U16, "mlp")
    h1 = product(b.o8, 1, gate=mod[2], residual=f64(h0))
    h2 = product(b.u8, 3, gate=mod[5], residual=h1)
    assert_elementwise(f64(b.h), h2, 2.0 ** -11 * (1 + np.abs(h2).max()), U32, "h")
    # and the whole against the block without any rounding: four products, whose operands' e4m3
    # roundings (2^-4 / sqrt 3 in the mean at most, on both) leave some 5% each of what is added
    full = [f64(w).T for w in b.full]
    xr = B.ln_modulate(f64(h0), mod[0], mod[1]) @ full[0].T + bias[0]
    q, k = (B.heads(xr[:, i * H:(i + 1) * H], HEADS, f64(b.pos), f64(b.freqs), SECTIONS, norm="rms_row", weight=f64(w))
            for i, w in enumerate((b.q_weight, b.k_weight)))
    v = xr[:, 2 * H:].reshape(tokens, HEADS, D).transpose(1, 0, 2)
    o = np.concatenate([O.attention(q[i], k[i], v[i]) for i in range(HEADS)], 1)
    hr = f64(h0) + mod[2] * (o @ full[1].T + bias[1])
    ur = B.linear(B.ln_modulate(hr, mod[3], mod[4]), full[2], bias[2], gelu=True)
    hr = hr + mod[5] * (ur @ full[3].T + bias[3])
    assert rel_err(f64(b.h) - f64(h0), hr - f64(h0)) < 0.2


@pytest.mark.parametrize("own_workspace", [False, True])
def test_captured_and_replayed(own_workspace):
    """The graph of a block, replayed over several inputs with eager work in between, gives the eager
    results' bits; two graphs that share one workspace, too."""
    P = need_gpu()
    a, c, eager = Block(P, 70, 6, 1), Block(P, 130, 10, 2), Block(P, 70, 6, 1)
    ws = torch.empty(max(1, a.workspace(), c.workspace()), dtype=torch.uint8, device="cuda") if own_workspace else None
    side = torch.cuda.Stream()
    graphs = []
    for b in (a, c):
        b.h.copy_(normal((b.L, H), 1))
        with torch.cuda.stream(side):
            b.run(workspace=ws)  # what is made once is made before the capture
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            b.run(workspace=ws)
        graphs.append(g)
    for i in range(4):
        h, h2 = normal((70, H), [7, i]), normal((130, H), [8, i])
        a.h.copy_(h)
        c.h.copy_(h2)
        graphs[0].replay()
        graphs[1].replay()
        eager.h.copy_(h)
        eager.run()
        torch.cuda.synchronize()
        assert _same(a.state(), eager.state())
        c2 = c.state()
        c.h.copy_(h2)
        c.run()
        assert _same(c2, c.state())


def test_streams_at_once():
    P = need_gpu()
    blocks = [Block(P, 130, 10, 3) for _ in range(3)]
    hs = [normal((130, H), [9, i]) for i in range(3)]
    want = []
    for b, h in zip(blocks, hs):
        b.h.copy_(h)
        b.run()
        want.append(b.state())
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(3):
        for b, h in zip(blocks, hs):
            b.h.copy_(h)
        torch.cuda.synchronize()
        for b, s in zip(blocks, streams):  # the stream given, and not the current one
            b.run(stream=s)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert _same(b.state(), w)
