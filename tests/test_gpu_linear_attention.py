"""Linear attention with per-head decay against its definition in 64 bits.

Bounds, per element.  An output is a sum of products whose factors are exact
or fp32; with A the same sum over absolute values, fp32 accumulation over L
tokens and d columns in any order, the decays' own roundings and a bf16
operand kept as two parts (relative error 2^-16) stay below
((L + d + 200) 2^-24 + 2^-15 [bf16]) A; a bf16 output adds half a step, 2^-8 of
its value.  A state is the same sum without the two-part operands.
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import assert_elementwise, need_gpu
from oracle import linear_block as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(t):
    return t.detach().double().cpu().numpy()


class Prompt:
    """Inputs on the device; vt's columns past L and all tokens past a
    sequence's length hold NaN, o a sentinel."""

    def __init__(self, dtype, n, heads, L, d, lengths=None, carried=True, slopes=None, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rnd(*s):
            return torch.randn(s, generator=g, device="cuda")

        self.n, self.heads, self.L, self.d, self.dt = n, heads, L, d, DT[dtype]
        self.len = [L] * n if lengths is None else [min(max(x, 0), L) for x in lengths]
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.q, self.k = rnd(n, heads, L, d).to(self.dt), rnd(n, heads, L, d).to(self.dt)
        self.vt = torch.full((n, heads, d, (L + 7) // 8 * 8 + 8), math.nan, device="cuda").to(self.dt)
        self.vt[..., :L] = rnd(n, heads, d, L).to(self.dt)
        for b, m in enumerate(self.len):
            self.q[b, :, m:], self.k[b, :, m:], self.vt[b, :, :, m:] = math.nan, math.nan, math.nan
        if slopes is None:
            slopes = [0.0 if h == 0 else 2.0 ** -(h % 9) for h in range(heads)]
        self.slopes = torch.tensor(slopes, dtype=torch.float32, device="cuda")
        self.state = rnd(n, heads, d, d) if carried else None
        self.o = torch.full((n, L, heads * d), 7.0, device="cuda").to(self.dt)
        self.state_out = torch.full((n, heads, d, d), 5.0, device="cuda")

    def run(self, P, **kw):
        P.linear_attention(self.q, self.k, self.vt, self.slopes, self.o, state_in=self.state,
                           state_out=self.state_out, lengths=self.lengths, **kw)
        return self

    def reference(self, scale, absolute=False):
        f = np.abs if absolute else (lambda x: x)
        for b, m in enumerate(self.len):
            v = _f64(self.vt[b])[:, :, :m].transpose(0, 2, 1)
            yield B.linear_attention(f(_f64(self.q[b])[:, :m]), f(_f64(self.k[b])[:, :m]), f(v),
                                     _f64(self.slopes),
                                     None if self.state is None else f(_f64(self.state[b])), scale)

    def check(self, scale=None, what=""):
        scale = self.d ** -0.5 if scale is None else scale
        bf16 = self.dt == torch.bfloat16
        acc = (self.L + self.d + 200) * 2.0 ** -24
        o, st = _f64(self.o), _f64(self.state_out)
        for b, ((ro, rs), (ao, as_)) in enumerate(zip(self.reference(scale),
                                                      self.reference(abs(scale), True))):
            m = self.len[b]
            assert_elementwise(o[b, :m], ro, (acc + (2.0 ** -15 if bf16 else 0)) * ao + 1e-35,
                               2.0 ** -8 if bf16 else 2.0 ** -24, f"{what} o[{b}]")
            assert_elementwise(st[b], rs, acc * as_ + 1e-35, 0.0, f"{what} state[{b}]")
            assert (o[b, m:] == 7.0).all(), "rows past the sequence's end were written"


CASES = [  # n, heads, L, d, lengths
    (1, 2, 1, 64, None), (1, 2, 1, 128, None), (2, 1, 2, 128, [2, 1]), (1, 3, 17, 128, None),
    (1, 1, 63, 64, None), (1, 2, 64, 128, None), (1, 2, 65, 64, None), (2, 2, 100, 128, [0, 100]),
    (3, 2, 129, 64, [129, 64, 65]), (2, 2, 200, 128, [-5, 1000]), (1, 3, 511, 64, None),
    (1, 2, 777, 128, None), (4, 1, 1100, 64, [1100, 1, 512, 1025]), (1, 2, 2500, 128, None),
    (1, 1, 3001, 64, None), (2, 1, 4100, 128, [4100, 2049]), (1, 2, 256, 128, None),
         (1, 2, 257, 64, None), (2, 8, 620, 64, [620, 301]), (4, 5, 640, 128, [640, 128, 129, 513])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,heads,L,d,lengths", CASES)
def test_prompts(dtype, n, heads, L, d, lengths):
    P = need_gpu()
    Prompt(dtype, n, heads, L, d, lengths, seed=L).run(P).check(what=f"{dtype} {n}x{heads}x{L}x{d}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,d", [(5, 64), (300, 128), (2100, 64)])
def test_from_no_state_and_with_a_scale(dtype, L, d):
    P = need_gpu()
    Prompt(dtype, 1, 2, L, d, carried=False, seed=1).run(P, scale=-0.3).check(-0.3)


@pytest.mark.parametrize("L", [9, 200, 2300])
def test_extreme_decays(L):
    """No decay, hardly any, total within a chunk, total at once, infinite."""
    P = need_gpu()
    Prompt("bf16", 1, 6, L, 64, slopes=[0.0, 1e-7, 1.5, 40.0, 3e38, math.inf], seed=2).run(P).check()
    Prompt("f32", 1, 4, L, 128, slopes=[0.0, 1e-6, 90.0, math.inf], seed=3).run(P).check()


def test_empty_sequences_hand_their_state_on():
    P = need_gpu()
    for lengths in (None, [0, -1]):
        for carried in (True, False):
            p = Prompt("bf16", 2, 2, 0 if lengths is None else 70, 64, lengths, carried).run(P)
            want = p.state if carried else torch.zeros_like(p.state_out)
            assert torch.equal(p.state_out, want)
            assert (p.o == 7.0).all()


@pytest.mark.parametrize("L", [40, 1500])
def test_no_state_wanted(L):
    P = need_gpu()
    a, b = (Prompt("bf16", 2, 2, L, 64, [L, L // 2], seed=4) for _ in range(2))
    a.run(P)
    b.state_out = None
    b.run(P)
    assert torch.equal(a.o, b.o)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,d", [(30, 128), (900, 64), (3000, 128)])
def test_state_in_place_and_repeatable(dtype, L, d):
    P = need_gpu()
    a, b, c = (Prompt(dtype, 2, 2, L, d, [L, L - 7], seed=5) for _ in range(3))
    a.run(P)
    b.state_out = b.state
    b.run(P)
    assert torch.equal(a.o, b.o) and torch.equal(a.state_out, b.state_out)
    ws = torch.full((max(P.linear_attention_workspace(2, 2, L, d), 1),), 255, dtype=torch.uint8,
                    device="cuda")
    c.run(P, workspace=ws)
    assert torch.equal(a.o, c.o) and torch.equal(a.state_out, c.state_out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("carried", [True, False])
@pytest.mark.parametrize("n,heads,L,d,lengths", [
    (1, 2, 65, 64, None), (2, 3, 128, 128, [127, 64]), (2, 2, 192, 64, [192, 0]), (3, 4, 320, 128, [320, 1, 65]),
    (1, 40, 500, 64, None), (5, 20, 511, 128, [511, 256, 0, 129, 64]), (13, 10, 513, 64, [513 - 40 * i for i in range(13)]),
    (4, 50, 260, 128, [260, 64, 0, 193])])
def test_segments_that_make_their_own_states(dtype, carried, n, heads, L, d, lengths):
    """With a state apart and in place, which shorter sequences take in
    different ways."""
    P = need_gpu()
    p = Prompt(dtype, n, heads, L, d, lengths, carried=carried, seed=L).run(P)
    p.check(what="apart")
    if carried:
        p.state_out, p.o = p.state.clone(), torch.full_like(p.o, 7.0)
        p.state, first = p.state_out, p.state
        p.run(P)
        p.state = first
        p.check(what="in place")


def test_later_tokens_do_not_reach_earlier_outputs():
    P = need_gpu()
    a, b = (Prompt("bf16", 1, 2, 500, 128, seed=6) for _ in range(2))
    for t in (b.q, b.k):
        t[:, :, 301:] = 100.0
    b.vt[..., 301:500] = -100.0
    assert torch.equal(a.run(P).o[:, :301], b.run(P).o[:, :301])


def test_many_sequences_and_heads():
    P = need_gpu()
    Prompt("bf16", 40, 9, 130, 64, [(37 * i) % 131 for i in range(40)], seed=7).run(P).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cut", [1, 64, 640])
def test_a_prompt_in_two_calls(dtype, cut):
    """The state carries: two calls and one differ by rounding alone."""
    P = need_gpu()
    p = Prompt(dtype, 1, 2, 1300, 64, seed=8).run(P)
    st = p.state.clone()
    o = torch.empty_like(p.o)
    for lo, hi in ((0, cut), (cut, 1300)):
        vt = torch.zeros((1, 2, 64, (hi - lo + 7) // 8 * 8), dtype=p.dt, device="cuda")
        vt[..., :hi - lo] = p.vt[..., lo:hi]
        part = torch.empty((1, hi - lo, 128), dtype=p.dt, device="cuda")
        P.linear_attention(p.q[:, :, lo:hi].contiguous(), p.k[:, :, lo:hi].contiguous(), vt,
                           p.slopes, part, state_in=st, state_out=st)
        o[:, lo:hi] = part
    p.o, p.state_out = o, st
    p.check(what="two calls")


def test_three_axes_are_one_sequence():
    P = need_gpu()
    p = Prompt("bf16", 1, 3, 77, 64, seed=9).run(P)
    o, st = torch.empty_like(p.o[0]), torch.empty_like(p.state_out[0])
    P.linear_attention(p.q[0], p.k[0], p.vt[0], p.slopes, o, state_in=p.state[0], state_out=st)
    assert torch.equal(o, p.o[0]) and torch.equal(st, p.state_out[0])


# ---------------------------------------------------------- single tokens


def _step_reference(q, k, v, slopes, state, slots, scale, n_slots):
    """Row by row; returns (o, states, absolute sums of both)."""
    heads, d = state.shape[1:3]
    S, A = state.copy(), np.abs(state)
    o, ao = np.full(q.shape, 7.0), np.zeros(q.shape)
    lam = np.exp(-slopes)[:, None, None]
    for r, s in enumerate(slots):
        if not 0 <= s < n_slots:
            continue
        qr, kr, vr = (x[r].reshape(heads, d) for x in (q, k, v))
        S[s] = lam * S[s] + kr[:, :, None] * vr[:, None, :]
        A[s] = lam * A[s] + np.abs(kr[:, :, None] * vr[:, None, :])
        o[r] = scale * np.einsum("hi,hij->hj", qr, S[s]).reshape(-1)
        ao[r] = abs(scale) * np.einsum("hi,hij->hj", np.abs(qr), A[s]).reshape(-1)
    return o, S, ao, A


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,d,n_slots,slots", [
    (1, 2, 64, 1, None), (1, 3, 128, 1, None), (5, 2, 128, 7, None),
    (4, 1, 64, 9, [8, 0, 3, 5]), (5, 2, 128, 4, [-1, 2, 4, 0, -2147483648]),
    (6, 2, 64, 3, [1, 0, 1, 1, -1, 0]), (3, 1, 128, 2, [-1, -1, 7]),
    (300, 1, 64, 290, "many")])
@pytest.mark.parametrize("in_place", [True, False])
def test_step(dtype, rows, heads, d, n_slots, slots, in_place):
    P = need_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows * 100 + d)
    if slots == "many":  # pairs and triples of rows far apart share a slot
        slots = [(i * 7) % 290 if i % 11 else -i for i in range(300)]
    w = heads * d
    qkv = torch.randn((rows, 3 * w + 8), generator=g, device="cuda").to(DT[dtype])
    q, k, v = (qkv[:, i * w:(i + 1) * w] for i in range(3))
    slopes = torch.rand(heads, generator=g, device="cuda")
    state = torch.randn((n_slots, heads, d, d), generator=g, device="cuda")
    wide = torch.full((rows, w + 16), 7.0, device="cuda").to(DT[dtype])
    o = wide[:, 8:8 + w]
    dev_slots = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
    names = slots if slots is not None else list(range(rows))
    ro, rs, ao, as_ = _step_reference(*(_f64(x) for x in (q, k, v, slopes, state)), names, 0.25,
                                      n_slots)
    out = state.clone() if in_place else torch.full_like(state, 5.0)
    if in_place:
        P.linear_attention_step(q, k, v, slopes, o, out, slots=dev_slots, scale=0.25)
    else:
        P.linear_attention_step(q, k, v, slopes, o, state, state_out=out, slots=dev_slots, scale=0.25)
        named = np.array([s in names for s in range(n_slots)])
        rs[~named] = 5.0
    acc = (d + 16 + max(names.count(s) for s in names)) * 2.0 ** -24
    bf16 = dtype == "bf16"
    assert_elementwise(_f64(o), ro, acc * ao, 2.0 ** -8 if bf16 else 2.0 ** -24, "o")
    assert_elementwise(_f64(out), rs, acc * as_, 0.0, "state")
    assert (wide[:, :8] == 7.0).all() and (wide[:, 8 + w:] == 7.0).all()


@pytest.mark.parametrize("rows", [1023, 1024, 1025, 5000])
def test_slots_far_apart(rows):
    """A slot's rows on both sides of the search's strides, among padding rows
    that are left alone."""
    P = need_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    where = {0: 5, 17: 9, 63: 2, 64: 2, 1022: 9, 1023: 5, 1024: 5, 1025: 2, 1041: 9, 2047: 3, 2048: 3,
             2111: 3, 3100: 11, 4990: 9, 4999: 5}
    slots = [where.get(r, -1) for r in range(rows)]
    q, k, v = (torch.randn((rows, 64), generator=g, device="cuda") for _ in range(3))
    slopes, state = torch.full((1,), 0.25, device="cuda"), torch.randn((16, 1, 64, 64), generator=g, device="cuda")
    ro, rs, ao, as_ = _step_reference(*(_f64(x) for x in (q, k, v, slopes, state)), slots, 0.5, 16)
    o = torch.full_like(q, 7.0)
    P.linear_attention_step(q, k, v, slopes, o, state, scale=0.5,
                            slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    acc = (64 + 16 + 5) * 2.0 ** -24
    assert_elementwise(_f64(o), ro, acc * ao, 2.0 ** -24, "o")
    assert_elementwise(_f64(state), rs, acc * as_, 0.0, "state")


def test_steps_follow_a_prompt():
    """A prompt, then tokens one by one, against the whole sequence."""
    P = need_gpu()
    p = Prompt("f32", 2, 2, 150, 64, carried=False, seed=11).run(P)
    q, k, vt = p.q[:, :, :140].contiguous(), p.k[:, :, :140].contiguous(), p.vt[..., :144].contiguous()
    st = torch.empty_like(p.state_out)
    P.linear_attention(q, k, vt, p.slopes, p.o[:, :140].contiguous(), state_out=st)
    for t in range(140, 150):
        row = [x[:, :, t].contiguous().reshape(2, 128) for x in (p.q, p.k, p.vt[..., :150].transpose(2, 3))]
        o = torch.empty_like(row[0])
        P.linear_attention_step(*row, p.slopes, o, st)
        p.o[:, t] = o
    p.state_out = st
    p.check(what="prompt + steps")


# ------------------------------------------------------ streams and graphs


def test_on_another_stream():
    P = need_gpu()
    want = Prompt("bf16", 1, 2, 1500, 64, seed=12).run(P)
    s = torch.cuda.Stream()
    p = Prompt("bf16", 1, 2, 1500, 64, seed=12)
    torch.cuda.synchronize()
    p.run(P, stream=s)
    s.synchronize()
    assert torch.equal(p.o, want.o) and torch.equal(p.state_out, want.state_out)
    with torch.cuda.stream(s):
        p.o.zero_()
        p.run(P)
    s.synchronize()
    assert torch.equal(p.o, want.o)


def test_captured_calls_replay():
    """Two graphs of two sizes, replayed in turn with eager work between;
    every replay against the eager result."""
    P = need_gpu()
    ps = [Prompt("bf16", 1, 2, L, 64, seed=13 + L) for L in (1500, 2600)]
    st = torch.randn((4, 2, 64, 64), device="cuda")
    row = torch.randn((3, 3, 128), device="cuda").bfloat16()
    slots = torch.tensor([2, 0, -1], dtype=torch.int32, device="cuda")
    slopes, so, sout = ps[0].slopes, torch.zeros(3, 128, device="cuda").bfloat16(), torch.zeros_like(st)

    def work(p):
        p.run(P)
        P.linear_attention_step(row[0], row[1], row[2], slopes, so, st, state_out=sout, slots=slots)

    graphs, want = [], []
    for p in ps:
        work(p)
        torch.cuda.synchronize()
        want.append((p.o.clone(), p.state_out.clone(), so.clone(), sout.clone()))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            work(p)
        graphs.append(g)
    for turn in range(3):
        for p, g, w in zip(ps, graphs, want):
            for t in (p.o, p.state_out, so, sout):
                t.zero_()
            torch.randn(1 << 20, device="cuda").sum()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for got, ref in zip((p.o, p.state_out, so, sout), w):
                assert torch.equal(got, ref), turn
