"""rotary_qkv of one token, and of one head, in place and through every view of them that torch has."""
import pytest
import torch

from fp8_util import normal
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _freqs(n):
    return torch.tensor([100.0 ** (-i / n) for i in range(n)], dtype=torch.float64, device="cuda")


@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
@pytest.mark.parametrize("tokens,heads,kv,n_seq", [(1, 6, 2, 1), (1, 1, 1, 1), (1, 6, 2, 3), (37, 1, 1, 1), (37, 1, 1, 2), (1, 1, 1, 3)])
def test_in_place(tokens, heads, kv, n_seq, pairs):
    P = need_gpu()
    d, rows = 64, n_seq * tokens
    wide = normal((rows, (heads + kv) * d + 64), [rows, heads], dtype=BF16)
    pos = torch.arange(5, 5 + rows, dtype=torch.int32, device="cuda")[None]
    args = (pos, _freqs(32), (32,))
    kw = dict(pairs=pairs, norm="rms")
    want = [torch.zeros((n_seq, h, tokens, d), dtype=BF16, device="cuda") for h in (heads, kv)]
    P.rotary_qkv(wide[:, :heads * d], wide[:, heads * d:(heads + kv) * d], None, *args, *want, None, **kw)
    for strided in (False, True):
        for lead in ((True, False) if n_seq == 1 else (True,)):
            mine = wide.clone()
            q, k = mine[:, :heads * d], mine[:, heads * d:(heads + kv) * d]
            if not strided:
                q, k = q.contiguous(), k.contiguous()
            views = []
            for t, h in ((q, heads), (k, kv)):
                if tokens == 1:   # the heads of a token as they lie in its row
                    view = t.unflatten(1, (h, 1, d))
                    assert view.stride(2) != t.stride(0) or h == 1
                else:             # one head: the rows themselves
                    view = t.unflatten(0, (n_seq, tokens)).unsqueeze(1)
                views.append(view if lead else view[0])
            P.rotary_qkv(q, k, None, *args, *views, None, **kw)
            for v, w in zip(views, want):
                assert torch.equal(v if lead else v[None], w)
            if strided:
                assert torch.equal(mine[:, (heads + kv) * d:], wide[:, (heads + kv) * d:])


def test_strides_that_nothing_depends_on():
    P = need_gpu()
    d = 64
    q, v = normal((1, 3 * d), 1, dtype=BF16), normal((1, 3 * d), 2, dtype=BF16)
    args = (torch.tensor([7], dtype=torch.int32, device="cuda"), _freqs(32), (32,))
    want, vt = torch.zeros((3, 1, d), dtype=BF16, device="cuda"), torch.zeros((3, d, 1), dtype=BF16, device="cuda")
    P.rotary_qkv(q, None, v, *args, want, None, vt)
    for stride in (0, 1, 7, 64, 1000):
        buf, vbuf = torch.full((4 * d,), 9.0, device="cuda").to(BF16), torch.zeros(3 * d, device="cuda").to(BF16)
        out = buf.as_strided((3, 1, d), (d, stride, 1))
        P.rotary_qkv(q, None, v, *args, out, None, vbuf.as_strided((3, d, 1), (d, 1, stride)))
        assert torch.equal(out, want) and (buf[3 * d:] == 9.0).all() and torch.equal(vbuf.view(3, d, 1), vt)
    for shape, strides in (((1, 3, 1, d), (5, d, 3, 1)), ((1, 3, 1, d), (0, d, 0, 1))):
        buf = torch.zeros(3 * d, device="cuda").to(BF16)
        P.rotary_qkv(q, None, None, *args, buf.as_strided(shape, strides), None, None)
        assert torch.equal(buf.view(3, 1, d), want)
