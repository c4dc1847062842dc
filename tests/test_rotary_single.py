"""rotary_qkv's checks where an axis has one entry: its stride, which no address depends on, may be
anything.  Calls that pass are seen by the refusal that comes last, of too many workgroups: nothing is
launched here."""
import ctypes as C

import pytest

from paper_2607_12358_amd import _lib as L

G = 1 << 44
# as many workgroups as are refused: V of 2^20 sequences of one token with 8 heads, or of 2^29 tokens
ONE_TOKEN, ONE_HEAD = dict(n_seq=1 << 20, tokens=1, heads=4, kv_heads=8), dict(n_seq=1, tokens=1 << 29, heads=1, kv_heads=1)


def _call(n_seq, tokens, heads, kv_heads, d=64, **kw):
    lib, a = L.lib(), L.RotaryQkvArgsC()
    v = dict(q=G, k=2 * G, v=3 * G, q_ld=heads * d, k_ld=kv_heads * d, v_ld=kv_heads * d, q_out=4 * G, k_out=5 * G, vt=6 * G,
             q_head=tokens * d, q_row=d, q_seq=heads * tokens * d, k_head=tokens * d, k_row=d, k_seq=kv_heads * tokens * d,
             vt_head=tokens * d, vt_row=tokens, vt_seq=kv_heads * tokens * d, positions=7 * G, positions_ld=n_seq * tokens,
             freqs=8 * G, in_dtype=L.ACID_BF16, out_dtype=L.ACID_BF16, heads=heads, kv_heads=kv_heads, head_dim=d, axes=1,
             q_scale=1.0, eps=1e-6)
    for key, x in {**v, **kw}.items():
        setattr(a, key, x)
    a.sections[:] = [32, 0, 0, 0]
    return lib.acid_rotary_qkv(C.byref(a), n_seq, tokens, None), L.last_error()


def test_the_last_refusal():
    for case in (ONE_TOKEN, ONE_HEAD):
        status, words = _call(**case)
        assert status == L.ACID_ERR_SHAPE and "workgroups" in words


@pytest.mark.parametrize("case,kw", [
    (ONE_TOKEN, dict(q_out=G)), (ONE_TOKEN, dict(k_out=2 * G)),      # rows as [n_seq, heads, 1, d]: in place
    (ONE_TOKEN, dict(q_out=G, q_row=0)), (ONE_TOKEN, dict(q_out=G, q_row=4 * 64)), (ONE_TOKEN, dict(q_out=G, q_row=1)),
    (ONE_TOKEN, dict(k_row=1)), (ONE_TOKEN, dict(k_row=0)), (ONE_TOKEN, dict(q_row=7)),
    (ONE_TOKEN, dict(q_out=G, q_ld=1024, q_seq=1024)),
    (ONE_HEAD, dict(q_out=G)), (ONE_HEAD, dict(q_out=G, q_head=0)), (ONE_HEAD, dict(q_out=G, q_ld=640, q_row=640)),
    (ONE_HEAD, dict(k_head=0)), (ONE_HEAD, dict(k_head=1)), (ONE_HEAD, dict(vt_head=1)),
    (dict(n_seq=1 << 20, tokens=1, heads=1, kv_heads=8), dict(q_out=G, q_row=1, q_head=1))])
def test_strides_of_one_entry(case, kw):
    status, words = _call(**case, **kw)
    assert status == L.ACID_ERR_SHAPE and "workgroups" in words, words


@pytest.mark.parametrize("case,kw,why", [
    (ONE_TOKEN, dict(q_out=G, q_seq=8 * 64), "overlaps an input"), (ONE_TOKEN, dict(q_out=G, q_ld=512), "overlaps an input"),
    (ONE_TOKEN, dict(q_out=G + 128), "overlaps an input"), (ONE_TOKEN, dict(q_out=G, q_head=128, q_seq=448), "overlaps an input"),
    (ONE_TOKEN, dict(q_out=G, out_dtype=L.ACID_F32), "overlaps an input"), (ONE_TOKEN, dict(q_seq=4 * 64 - 8), "values apart"),
    (ONE_TOKEN, dict(q_head=0), "values apart"), (ONE_TOKEN, dict(k_out=4 * G + 256), "outputs overlap"),
    (ONE_HEAD, dict(q_out=G, q_row=128), "overlaps an input"), (ONE_HEAD, dict(q_row=60), "values apart")])
def test_what_stays_refused(case, kw, why):
    status, words = _call(**case, **kw)
    assert status in (L.ACID_ERR_SHAPE, L.ACID_ERR_INVALID_ARG) and why in words, words
