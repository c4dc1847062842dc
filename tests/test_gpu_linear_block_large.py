"""The linear-attention block's entry points past 32-bit offsets, at once on two
streams, and with one workspace for two graphs."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu
from oracle import linear_block as B

pytestmark = pytest.mark.gpu


def _rand(*shape, dtype=torch.float32, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def test_state_pool_past_4_gib():
    """Slots on both sides of 2^32 bytes and of 2^31 values, against a small
    pool with the same states: the same bits."""
    P = need_gpu()
    n, heads, d = 11000, 12, 128  # 8.6 GB
    pool = torch.zeros((n, heads, d, d), device="cuda")
    slots = [0, 5461, 5462, 10923, 10999]
    small = _rand(5, heads, d, d, seed=1)
    pool[slots] = small
    q, k, v = (_rand(5, heads * d, dtype=torch.bfloat16, seed=s) for s in (2, 3, 4))
    sl = torch.full((heads,), 0.1, device="cuda")
    o, want = torch.empty_like(q), torch.empty_like(q)
    P.linear_attention_step(q, k, v, sl, o, pool,
                            slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    P.linear_attention_step(q, k, v, sl, want, small)
    assert torch.equal(o, want) and torch.equal(pool[slots], small)
    assert float(pool[1].abs().sum()) == 0.0 and float(pool[10998].abs().sum()) == 0.0


def test_prompt_past_2_31_values():
    """The last of 32 heads of 550000 tokens (2.25e9 values a tensor), against
    the same head by itself.  Both are within 2^-15 of the sum of absolute
    products of the exact outputs, and bf16 rounding; a wrong offset is off by
    the outputs' own scale."""
    P = need_gpu()
    heads, L, d = 32, 550000, 128
    q, k = (_rand(heads, L, d, dtype=torch.bfloat16, seed=s) for s in (1, 2))
    vt = _rand(heads, d, L, dtype=torch.bfloat16, seed=3)
    sl = torch.full((heads,), 0.02, device="cuda")
    o = torch.empty((L, heads * d), dtype=torch.bfloat16, device="cuda")
    st = torch.empty((heads, d, d), device="cuda")
    P.linear_attention(q, k, vt, sl, o, state_out=st)
    for h in (0, 16, 31):
        o1 = torch.empty((L, d), dtype=torch.bfloat16, device="cuda")
        st1 = torch.empty((1, d, d), device="cuda")
        P.linear_attention(q[h:h + 1], k[h:h + 1], vt[h:h + 1], sl[:1], o1, state_out=st1)
        a, b = o[:, h * d:(h + 1) * d].float(), o1.float()
        rms = float(b.square().mean().sqrt())
        assert float(((a - b).abs() - 2.0 ** -7 * b.abs()).max()) <= 0.02 * rms, h
        assert float((st[h] - st1[0]).abs().max()) <= 1e-4 * float(st1.square().mean().sqrt()), h


def test_seam_past_2_31_values():
    """Rows on both sides of 2^31 values, against those rows by themselves:
    the same bits."""
    P = need_gpu()
    rows, hidden = 530000, 4096
    h = torch.zeros((rows, hidden), device="cuda")
    y = torch.zeros((rows, hidden), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((rows, hidden), dtype=torch.bfloat16, device="cuda")
    pick = [0, 262143, 262144, 524287, 524288, 529999]
    h[pick], y[pick] = _rand(6, hidden, seed=1), _rand(6, hidden, dtype=torch.bfloat16, seed=2)
    hs, ys, os_ = h[pick].clone(), y[pick].clone(), torch.empty((6, hidden), dtype=torch.bfloat16,
                                                                device="cuda")
    g = _rand(hidden, seed=3)
    P.residual_norm(h, y, out=out, post="rms", gate=g, pre="layer")
    P.residual_norm(hs, ys, out=os_, post="rms", gate=g, pre="layer")
    assert torch.equal(h[pick], hs) and torch.equal(out[pick], os_)


def test_w4_past_4_gib_of_codes():
    """The first and last tiles of 2^22 outputs of 2176 inputs (4.6 GB of
    codes), against the same tiles by themselves: the same bits."""
    P = need_gpu()
    n, k = 1 << 22, 2176
    cs, ss = P.w4_shapes(n, k, 128)
    codes = torch.full(cs, 0x88, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(ss, device="cuda")
    tiles = [0, 123361, 123362, 246723, 246724, cs[0] - 1]  # around 2^31 and 2^32 bytes
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    some = torch.randint(0, 256, (6,) + cs[1:], generator=g, device="cuda", dtype=torch.uint8)
    scale = _rand(6, *ss[1:], seed=5)
    codes[tiles], scales[tiles] = some, scale
    x = _rand(2, k, seed=6)
    out, want = torch.empty((2, n), device="cuda"), torch.empty((2, 96), device="cuda")
    P.linear_w4(x, codes, scales, out)
    P.linear_w4(x, some, scale, want)
    got = torch.cat([out[:, 16 * t:16 * t + 16] for t in tiles], 1)
    ref = B.linear_w4(x.double().cpu().numpy(), some.cpu().numpy(), scale.cpu().numpy(), 96)
    bound = 2.0 ** -15 * np.abs(x.double().cpu().numpy()).sum(1)[:, None] * 40 * float(scale.abs().max())
    assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()
    assert (np.abs(want.double().cpu().numpy() - ref) <= bound).all()
    assert float(out[:, 16:160].abs().max()) == 0.0


def test_two_calls_at_once():
    """The same call on two streams, each with the workspace it is given by
    default, over and over: every result is the one alone."""
    P = need_gpu()
    q, k = (_rand(2, 3, 2000, 64, dtype=torch.bfloat16, seed=s) for s in (1, 2))
    vt = _rand(2, 3, 64, 2000, dtype=torch.bfloat16, seed=3)
    sl = torch.tensor([0.0, 0.01, 0.5], device="cuda")
    st = _rand(2, 3, 64, 64, seed=4)

    def call(o, s, stream=None):
        P.linear_attention(q, k, vt, sl, o, state_in=st, state_out=s, stream=stream)

    outs = [(torch.empty((2, 2000, 192), dtype=torch.bfloat16, device="cuda"), torch.empty_like(st))
            for _ in range(9)]
    call(*outs[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(1, 9):
        call(*outs[i], stream=streams[i % 2])
    torch.cuda.synchronize()
    for o, s in outs[1:]:
        assert torch.equal(o, outs[0][0]) and torch.equal(s, outs[0][1])


def test_one_workspace_for_two_graphs():
    P = need_gpu()
    ws = torch.empty(max(P.linear_attention_workspace(1, 2, n, 64) for n in (3000, 1700)),
                     dtype=torch.uint8, device="cuda")
    sl = torch.tensor([0.0, 0.3], device="cuda")
    runs = []
    for n in (3000, 1700):
        q, k = (_rand(2, n, 64, dtype=torch.bfloat16, seed=n + s) for s in (1, 2))
        vt = torch.zeros((2, 64, (n + 7) // 8 * 8), dtype=torch.bfloat16, device="cuda")
        vt[..., :n] = _rand(2, 64, n, dtype=torch.bfloat16, seed=n)
        o, st = torch.empty((n, 128), dtype=torch.bfloat16, device="cuda"), torch.empty(2, 64, 64, device="cuda")
        call = lambda q=q, k=k, vt=vt, o=o, st=st: P.linear_attention(  # noqa: E731
            q, k, vt, sl, o, state_out=st, workspace=ws)
        call()
        torch.cuda.synchronize()
        want = (o.clone(), st.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        runs.append((g, o, st, want, call))  # call: a graph's inputs have to stay
    for _ in range(3):
        for g, o, st, want, _ in runs:
            o.zero_()
            st.zero_()
            ws.fill_(255)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want[0]) and torch.equal(st, want[1])
