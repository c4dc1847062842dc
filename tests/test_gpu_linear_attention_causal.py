"""A NaN or an infinity in one token reaches that token and the ones after it,
in its own head (and, from v, in its own column); all that comes before it, and
all other heads and columns, are the bits they are without it."""
import math

import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# dtype, sequences, heads, tokens, head_dim, token: first, last and inner ones of a chunk, ragged chunks, segments
# in each of their forms
CASES = [(dt, *c) for dt in ("bf16", "f32") for c in (
    (1, 2, 1, 64, 0), (1, 2, 17, 128, 9), (1, 2, 64, 64, 63), (2, 2, 64, 128, 31), (1, 2, 130, 64, 129),
    (1, 3, 200, 128, 80), (1, 2, 1000, 64, 500), (2, 8, 620, 128, 64 * 4 + 17), (1, 40, 500, 64, 200),
    (1, 2, 2500, 128, 1313))]


def _run(P, q, k, vt, slopes, state, in_place):
    n, heads, L, d = q.shape
    o = torch.empty((n, L, heads * d), dtype=q.dtype, device="cuda")
    out = state.clone() if in_place else torch.empty_like(state)
    P.linear_attention(q, k, vt, slopes, o, state_in=out if in_place else state, state_out=out)
    return o.view(n, L, heads, d), out


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,n,heads,L,d,at", CASES)
def test_one_token_that_is_not_finite(dtype, n, heads, L, d, at, bad):
    P = need_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(L)

    def rnd(*s):
        return torch.randn(s, generator=g, device="cuda")

    q, k = (rnd(n, heads, L, d).to(DT[dtype]) for _ in range(2))
    vt = rnd(n, heads, d, (L + 7) // 8 * 8).to(DT[dtype])
    slopes = torch.tensor([0.0, 0.02, 1.5] * heads, device="cuda")[:heads].contiguous()
    state = rnd(n, heads, d, d)
    b, h, c = n - 1, heads // 2, d - 3   # where it is
    for in_place in (False, True):
        o, st = _run(P, q, k, vt, slopes, state, in_place)
        for name in "vkq":
            q1, k1, vt1 = q.clone(), k.clone(), vt.clone()
            if name == "v":
                vt1[b, h, c, at] = bad
            else:
                (k1 if name == "k" else q1)[b, h, at, c] = bad
            o1, st1 = _run(P, q1, k1, vt1, slopes, state, in_place)
            spoilt, spoilt_state = torch.zeros_like(o, dtype=torch.bool), torch.zeros_like(st, dtype=torch.bool)
            if name == "v":
                spoilt[b, at:, h, c] = True
                spoilt_state[b, h, :, c] = True
            elif name == "k":
                spoilt[b, at:, h] = True
                spoilt_state[b, h, c] = True
            else:
                spoilt[b, at, h] = True
            what = (name, in_place)
            assert torch.equal(o1[~spoilt], o[~spoilt]), what
            assert torch.equal(st1[~spoilt_state], st[~spoilt_state]), what
            assert not torch.isfinite(o1[spoilt]).any(), what
            assert not torch.isfinite(st1[spoilt_state]).any(), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_columns_and_tokens(dtype):
    """Each column from its own first bad token on, in a padded batch."""
    P = need_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    n, heads, L, d = 3, 2, 150, 64
    q, k = (torch.randn((n, heads, L, d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    vt = torch.randn((n, heads, d, 152), generator=g, device="cuda").to(DT[dtype])
    lengths = torch.tensor([150, 100, 0], dtype=torch.int32, device="cuda")
    slopes = torch.tensor([0.0, 0.3], device="cuda")

    def run(v):
        o, st = torch.full((n, L, heads * d), 7.0, device="cuda").to(q.dtype), torch.empty((n, heads, d, d), device="cuda")
        P.linear_attention(q, k, v, slopes, o, state_out=st, lengths=lengths)
        return o.view(n, L, heads, d), st

    o, st = run(vt)
    bad = vt.clone()
    first = torch.full((n, heads, d), L, device="cuda")
    for b, h, c, t, x in ((0, 0, 0, 149, math.inf), (0, 0, 1, 3, math.nan), (0, 0, 1, 70, math.inf), (0, 1, 17, 64, -math.inf),
                          (0, 1, 63, 63, math.nan), (1, 0, 5, 99, math.nan), (1, 0, 6, 100, math.nan), (1, 1, 40, 20, math.inf),
                          (1, 1, 40, 21, -math.inf), (2, 0, 8, 0, math.nan)):
        bad[b, h, c, t] = x
        if t < int(lengths[b]):
            first[b, h, c] = min(int(first[b, h, c]), t)
    o1, st1 = run(bad)
    t = torch.arange(L, device="cuda")[None, :, None, None]
    spoilt = (t >= first[:, None]) & (t < lengths[:, None, None, None])
    spoilt_state = (first < L)[:, :, None, :].expand_as(st)
    assert torch.equal(o1[~spoilt], o[~spoilt]) and torch.equal(st1[~spoilt_state], st[~spoilt_state])
    assert not torch.isfinite(o1[spoilt]).any() and not torch.isfinite(st1[spoilt_state]).any()
