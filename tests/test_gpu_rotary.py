"""Heads with positions against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from fp8_util import U16, U32, f64, normal
from gpu_util import assert_elementwise, need_gpu
from oracle import fp8_block as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _freqs(n, theta=10000.0):
    return torch.tensor([theta ** (-i / max(n, 1)) for i in range(n)], dtype=torch.float64, device="cuda")


def _positions(axes, tokens, seed, most=100, dtype=torch.int32):
    p = np.random.default_rng(seed).integers(0, most, (axes, tokens))
    return torch.from_numpy(p).to(dtype).cuda()


def _bound(rows, heads, norm, weight, bias, scale, out_dtype):
    """A value is a sum of two products, each with some ten fp32 roundings (norm, weight, angle's
    sine, products) of the pair's largest parts, then one rounding to the output's type."""
    d = rows.shape[1] // heads
    x = np.abs(B.heads(rows, heads, np.zeros((1, rows.shape[0])), np.zeros(1), (0,), norm=norm))  # |normed|
    if norm == "layer":  # the mean is taken from the values
        x = x + 1
    w = 1.0 if weight is None else np.abs(weight).reshape((heads, 1, d) if norm == "rms_row" else (1, 1, d))
    b = 0.0 if bias is None else np.abs(bias)
    pair = (x * w + b).max(2, keepdims=True)  # of the head: of either pairing
    return abs(scale) * 48 * U32 * pair, U16 if out_dtype == BF16 else U32


def _check(got, rows, heads, pos, freqs, sections, pairs, norm, weight, bias, scale, what):
    want = B.heads(rows, heads, pos, freqs, sections, pairs, norm, weight, bias, scale)
    atol, rtol = _bound(rows, heads, norm, weight, bias, scale, got.dtype)
    assert_elementwise(f64(got), want, (1 + U16) * atol + 2.0 ** -133, rtol, what)


def _weights(norm, heads, kv, d):
    if norm == "none":
        return [None] * 4
    n = (heads * d, kv * d) if norm == "rms_row" else (d, d)
    return [normal(n[0], 1, 0.2, 1.0), normal(n[1], 2, 0.2, 1.0)] + (
        [normal(d, 3, 0.2), normal(d, 4, 0.2)] if norm == "layer" else [None, None])


@pytest.mark.parametrize("tokens,heads,kv,d,sections", [
    (1, 1, 1, 64, (32,)), (1, 16, 4, 64, (32,)), (1, 12, 12, 128, (22, 21, 21)), (7, 3, 3, 128, (16, 24, 24)),
    (15, 5, 1, 64, (8, 8)), (17, 2, 2, 64, (16, 8, 8)), (63, 4, 2, 128, (64,)), (64, 1, 1, 128, (0, 32, 32)),
    (65, 7, 7, 64, (8, 4, 4)), (130, 24, 8, 128, (8, 8, 8, 8)), (257, 40, 40, 128, (22, 21, 21)), (100, 33, 3, 64, (32,)),
    (3, 1024, 1024, 64, (12, 10, 10))])
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
@pytest.mark.parametrize("norm", ["none", "rms", "layer", "rms_row"])
@pytest.mark.parametrize("din,dout", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)], ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
def test_heads(tokens, heads, kv, d, sections, pairs, norm, din, dout):
    P = need_gpu()
    qkv = normal((tokens, (heads + 2 * kv) * d), [tokens, heads], 1.5, 0.3, din)
    q, k, v = qkv[:, :heads * d], qkv[:, heads * d:(heads + kv) * d], qkv[:, (heads + kv) * d:]
    n = sum(sections)
    pos, freqs = _positions(len(sections), tokens, tokens), _freqs(n)
    qw, kw, qb, kb = _weights(norm, heads, kv, d)
    qo = torch.full((heads, tokens, d), 9.0, device="cuda", dtype=dout)
    ko = torch.full((kv, tokens, d), 9.0, device="cuda", dtype=dout)
    ld = (tokens + 7) // 8 * 8
    whole = torch.full((kv, d, ld), 9.0, device="cuda", dtype=dout)
    scale = P.q_scale(d)
    P.rotary_qkv(q, k, v, pos, freqs, sections, qo, ko, whole[:, :, :tokens], pairs=pairs, norm=norm, q_weight=qw,
                 k_weight=kw, q_bias=qb, k_bias=kb, q_scale=scale)
    a = [None if t is None else f64(t) for t in (qw, kw, qb, kb)]
    common = (f64(pos), f64(freqs), sections, pairs, norm)
    _check(qo, f64(q), heads, *common, a[0], a[2], scale, "q")
    _check(ko, f64(k), kv, *common, a[1], a[3], 1.0, "k")
    vt = v.float().reshape(tokens, kv, d).permute(1, 2, 0).to(dout)
    assert torch.equal(whole[:, :, :tokens], vt) and (whole[:, :, tokens:] == 9.0).all()


def _some(P, tokens=37, heads=6, kv=2, d=64, dtype=BF16, seed=5):
    qkv = normal((tokens, (heads + 2 * kv) * d), seed, dtype=dtype)
    rows = qkv[:, :heads * d], qkv[:, heads * d:(heads + kv) * d], qkv[:, (heads + kv) * d:]
    outs = (torch.zeros((heads, tokens, d), dtype=dtype, device="cuda"), torch.zeros((kv, tokens, d), dtype=dtype, device="cuda"),
            torch.zeros((kv, d, tokens), dtype=dtype, device="cuda"))
    pos, sections = _positions(3, tokens, 3), (12, 10, 10)
    return qkv, rows, outs, pos, _freqs(32), sections


@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
def test_layouts_give_the_same_values(pairs):
    """Heads outermost, tokens outermost, in place, a cache's rows, sequences: the same bits."""
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, vt), pos, freqs, sections = _some(P)
    kw = dict(pairs=pairs, norm="rms")
    P.rotary_qkv(q, k, v, pos, freqs, sections, qo, ko, vt, **kw)
    # each alone
    for i in range(3):
        one = [torch.zeros_like(o) if j == i else None for j, o in enumerate((qo, ko, vt))]
        rows = [r if j == i else None for j, r in enumerate((q, k, v))]
        P.rotary_qkv(*rows, pos, freqs, sections, *one, **kw)
        assert torch.equal(one[i], (qo, ko, vt)[i])
    # tokens outermost
    tq, tk = torch.zeros(37, 6, 64, dtype=BF16, device="cuda"), torch.zeros(37, 2, 64, dtype=BF16, device="cuda")
    P.rotary_qkv(q, k, None, pos, freqs, sections, tq.transpose(0, 1), tk.transpose(0, 1), None, **kw)
    assert torch.equal(tq.transpose(0, 1), qo) and torch.equal(tk.transpose(0, 1), ko)
    # rows of caches, off 16 bytes in the transposed one
    for at in (0, 5, 8, 11):
        kc, vc = torch.full((2, 64, 64), 7.0, device="cuda").bfloat16(), torch.full((2, 64, 72), 7.0, device="cuda").bfloat16()
        P.rotary_qkv(None, k, v, pos, freqs, sections, None, kc[:, at:at + 37], vc[:, :, at:at + 37], **kw)
        assert torch.equal(kc[:, at:at + 37], ko) and torch.equal(vc[:, :, at:at + 37], vt)
        kc[:, at:at + 37], vc[:, :, at:at + 37] = 7.0, 7.0
        assert (kc == 7.0).all() and (vc == 7.0).all()
    # fp32 positions of whole numbers, and a row-strided matrix of them
    wide = torch.zeros(3, 50, dtype=torch.int32, device="cuda")
    wide[:, :37] = pos
    for p in (pos.float(), wide[:, :37]):
        again = [torch.zeros_like(t) for t in (qo, ko, vt)]
        P.rotary_qkv(q, k, v, p, freqs, sections, *again, **kw)
        assert all(torch.equal(x, y) for x, y in zip(again, (qo, ko, vt)))
    # two sequences whose tokens follow one another
    two = torch.cat((qkv, qkv.flip(0)))
    p2 = torch.cat((pos, pos.flip(1)), 1).contiguous()
    o2 = [torch.zeros((2, *t.shape), dtype=BF16, device="cuda") for t in (qo, ko, vt)]
    P.rotary_qkv(two[:, :384], two[:, 384:512], two[:, 512:], p2, freqs, sections, *o2, **kw)
    for x, y in zip(o2, (qo, ko, vt)):
        assert torch.equal(x[0], y)
        assert torch.equal(x[1], y.flip(2 if y is vt else 1))
    # in place, tokens outermost
    P.rotary_qkv(q, k, None, pos, freqs, sections, qkv.as_strided((6, 37, 64), (64, 640, 1)),
                 qkv.as_strided((2, 37, 64), (64, 640, 1), 384), None, **kw)
    assert torch.equal(qkv[:, :384].reshape(37, 6, 64).transpose(0, 1), qo)
    assert torch.equal(qkv[:, 384:512].reshape(37, 2, 64).transpose(0, 1), ko)
    assert torch.equal(qkv[:, 512:].reshape(37, 2, 64).permute(1, 2, 0), vt)


def test_one_buffer_for_both_caches():
    """K and V^T side by side for each head, or for each sequence: apart, though their reaches cross."""
    P = need_gpu()
    _, (q, k, v), (_, ko, vt), pos, freqs, sections = _some(P, tokens=37)
    P.rotary_qkv(None, k, v, pos, freqs, sections, None, ko, vt)
    cap, d = 48, 64
    for n_seq in (1, 2):
        rows = [torch.cat([t] * n_seq) for t in (k, v)]
        p = torch.cat([pos] * n_seq, 1).contiguous()
        for by_head in (True, False):
            head = (2 if by_head else 1) * cap * d
            seq = 4 * cap * d
            buf = torch.full((n_seq * seq,), 7.0, device="cuda").bfloat16()
            kc = buf.as_strided((n_seq, 2, 37, d), (seq, head, d, 1), 0)
            vc = buf.as_strided((n_seq, 2, d, 37), (seq, head, cap, 1), (1 if by_head else 2) * cap * d)
            P.rotary_qkv(None, *rows, p, freqs, sections, None, kc, vc)
            for s in range(n_seq):
                assert torch.equal(kc[s], ko) and torch.equal(vc[s], vt)
            left = buf.clone()
            left.as_strided(kc.shape, kc.stride(), kc.storage_offset()).fill_(7.0)
            left.as_strided(vc.shape, vc.stride(), vc.storage_offset()).fill_(7.0)
            assert (left == 7.0).all()
            with pytest.raises(P.AcidError, match="outputs overlap"):
                P.rotary_qkv(None, *rows, p, freqs, sections, None, kc, buf.as_strided(vc.shape, vc.stride(), 36 * d))


@pytest.mark.parametrize("norm", ["none", "rms_row"])
def test_in_place_rows_norm(norm):
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, _), pos, freqs, sections = _some(P, tokens=300, heads=24, kv=24, d=128, seed=8)
    freqs, sections = _freqs(64), (22, 21, 21)
    P.rotary_qkv(q, k, None, pos, freqs, sections, qo, ko, None, norm=norm)
    ld, h = qkv.stride(0), 24 * 128
    P.rotary_qkv(q, k, None, pos, freqs, sections, qkv.as_strided((24, 300, 128), (128, ld, 1)),
                 qkv.as_strided((24, 300, 128), (128, ld, 1), h), None, norm=norm)
    assert torch.equal(qkv[:, :h].reshape(300, 24, 128).transpose(0, 1), qo)
    assert torch.equal(qkv[:, h:2 * h].reshape(300, 24, 128).transpose(0, 1), ko)


def test_text_at_the_origin_is_not_turned():
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, vt), pos, freqs, sections = _some(P)
    pos[:, :10] = 0
    P.rotary_qkv(q, k, v, pos, freqs, sections, qo, ko, vt)
    assert torch.equal(qo[:, :10], q[:10].reshape(10, 6, 64).transpose(0, 1))
    assert not torch.equal(qo[:, 10:], q[10:].reshape(27, 6, 64).transpose(0, 1))


def test_far_and_fractional_positions():
    """Angles of positions to 2^31 - 1 keep their fraction of a turn; fractions and negative ones."""
    P = need_gpu()
    for dtype, values in ((torch.int32, [0, 1, 2 ** 20 + 1, 2 ** 31 - 1, -2 ** 31, -7, 123456789]),
                          (F32, [0.5, 0.25, -3.75, 1e-3, 65536.5, 2.0 ** 30, 12345.678])):
        pos = torch.tensor(values, dtype=dtype, device="cuda")
        q = normal((7, 128), 3)
        qo = torch.zeros(2, 7, 64, device="cuda")
        freqs = _freqs(32)
        P.rotary_qkv(q, None, None, pos, freqs, (32,), qo, None, None, pairs="halves")
        want = B.heads(f64(q), 2, f64(pos)[None], f64(freqs), (32,), "halves")
        # the angle itself is exact to 2^-52 of its size in 64 bits
        off = (48 * U32 + 4 * 2.0 ** -52 * np.abs(f64(pos))[None, :, None]) * np.abs(f64(q)).max()
        assert_elementwise(f64(qo), want, off, U32)


def test_what_is_not_finite_stays_in_its_pair():
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, vt), pos, freqs, sections = _some(P)
    freqs, sections = _freqs(16), (16, 0, 0)      # dims 32 on do not turn
    for pairs, partner in (("adjacent", 5), ("halves", 4 + 16)):
        clean = qo.clone()
        P.rotary_qkv(q, None, None, pos, freqs, sections, clean, None, None, pairs=pairs)
        dirty = q.clone()
        dirty[3, 64 + 4], dirty[3, 64 + 40] = float("nan"), float("inf")
        P.rotary_qkv(dirty, None, None, pos, freqs, sections, qo, None, None, pairs=pairs)
        bad = torch.zeros_like(qo, dtype=torch.bool)
        bad[1, 3, 4] = bad[1, 3, partner] = bad[1, 3, 40] = True
        assert torch.equal(~torch.isfinite(qo), bad) and torch.equal(qo[~bad], clean[~bad])


def test_no_pairs_and_no_tokens():
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, vt), *_ = _some(P)
    P.rotary_qkv(q, k, v, None, None, (0,), qo, ko, vt)
    assert torch.equal(qo, q.reshape(37, 6, 64).transpose(0, 1)) and torch.equal(vt, v.reshape(37, 2, 64).permute(1, 2, 0))
    P.rotary_qkv(q[:0], None, None, torch.zeros((1, 0), dtype=torch.int32, device="cuda"), _freqs(8), (8,), qo[:, :0], None, None)


def test_refusals():
    P = need_gpu()
    qkv, (q, k, v), (qo, ko, vt), pos, freqs, sections = _some(P)
    ok = dict(q=q, k=k, v=v, positions=pos, freqs=freqs, sections=sections, q_out=qo, k_out=ko, vt=vt)
    P.rotary_qkv(**ok)
    for kw in (dict(norm="l2"), dict(pairs="other"), dict(sections=()), dict(sections=(8,) * 5), dict(q=None), dict(vt=None),
               dict(q=q.float()), dict(k_out=ko.float()), dict(positions=pos.long()), dict(positions=pos[:2]),
               dict(freqs=freqs.float()), dict(freqs=freqs[:3]), dict(q_out=qo[:, :36]), dict(vt=vt.transpose(1, 2)),
               dict(q_weight=torch.ones(3, device="cuda"), norm="rms"), dict(q_out=qo.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            P.rotary_qkv(**{**ok, **kw})
    wide = torch.zeros(6, 37, 66, device="cuda").bfloat16()
    for kw, why in ((dict(sections=(20, 10, 10), freqs=_freqs(40)), "40 pairs"), (dict(sections=(5, 2, 2), freqs=_freqs(9), pairs="halves"), "9 pairs"),
                    (dict(q_weight=torch.ones(64, device="cuda")), "without a norm"), (dict(q_bias=torch.ones(64, device="cuda"), norm="rms",
                     q_weight=torch.ones(64, device="cuda")), "biases"), (dict(q_out=wide[..., :64]), "16 bytes"),
                    (dict(q_out=qkv.as_strided((6, 37, 64), (64, 640, 1), 64)), "overlap"), (dict(eps=-1.0), "eps"),
                    (dict(k_out=qo[:2]), "outputs overlap"), (dict(q_out=qo[:1].expand(6, 37, 64)), "values apart")):
        with pytest.raises(P.AcidError, match=why):
            P.rotary_qkv(**{**ok, **kw})
