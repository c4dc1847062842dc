"""Argument checks of the linear-attention block's entry points: every call
here is refused, or has nothing to do, before any GPU work (made-up addresses
are never looked at)."""
import ctypes as C

import pytest
import torch

import paper_2607_12358_amd as P
from paper_2607_12358_amd import _lib as L

BAD, SHAPE, UNSUPPORTED = L.ACID_ERR_INVALID_ARG, L.ACID_ERR_SHAPE, L.ACID_ERR_UNSUPPORTED
G = 1 << 30  # made-up buffers lie whole gigabytes apart


@pytest.fixture(scope="module")
def lib():
    return L.lib()


def _attend(lib, **kw):
    a = dict(dtype=L.ACID_BF16, n=2, heads=3, L=100, d=64, q=G, k=2 * G, vt=3 * G, ld=104,
             slopes=4 * G, lengths=None, sin=None, sout=None, scale=1.0, o=5 * G, ws=6 * G,
             bytes=1 << 40)
    a.update(kw)
    return lib.acid_linear_attention(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), BAD), (dict(n=-1), BAD), (dict(heads=0), BAD), (dict(L=-1), BAD),
    (dict(d=96), SHAPE), (dict(ld=96), SHAPE), (dict(ld=108), SHAPE), (dict(ld=1 << 33), SHAPE),
    (dict(n=1 << 21, heads=2), SHAPE), (dict(L=1 << 31, ld=1 << 31), SHAPE),
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(vt=None), BAD), (dict(o=None), BAD),
    (dict(slopes=None), BAD), (dict(q=G + 8), BAD), (dict(sin=7 * G + 4), BAD),
    (dict(o=G + 16), BAD), (dict(o=2 * G), BAD), (dict(o=3 * G), BAD), (dict(sout=5 * G), BAD),
    (dict(sin=5 * G), BAD), (dict(sout=G), BAD), (dict(sin=7 * G, sout=7 * G + 256), BAD)])
def test_attention_refusals(lib, kw, status):
    assert _attend(lib, **kw) == status
    assert L.last_error()


def test_attention_refuses_a_small_workspace(lib):
    need = lib.acid_linear_attention_workspace_bytes(1, 2, 40000, 128)
    if need:
        for ws, size in ((6 * G, need - 1), (None, 0), (6 * G + 8, need)):
            assert _attend(lib, n=1, heads=2, L=40000, ld=40000, d=128, ws=ws,
                           bytes=size) in (SHAPE, BAD)
    assert lib.acid_linear_attention_workspace_bytes(1, 2, 40000, 96) == 0
    assert lib.acid_linear_attention_workspace_bytes(1, 2, -1, 64) == 0


def test_workspace_needed_is_no_more_than_enough(lib):
    some = 0
    for dtype in (L.ACID_BF16, L.ACID_F32):
        for d in (64, 128):
            for heads in (1, 2, 5, 8, 31, 64, 65, 86, 100, 128, 129, 171, 256, 257, 384, 385, 1000):
                for tokens in (0, 1, 64, 65, 129, 300, 512, 1000, 3000, 5000, 40000, 1 << 28):
                    enough = lib.acid_linear_attention_workspace_bytes(1, heads, tokens, d)
                    in_place, apart = (lib.acid_linear_attention_workspace_needed(dtype, 1, heads, tokens, d, i)
                                       for i in (1, 0))
                    assert apart in (0, in_place) and in_place <= enough
                    assert enough % (heads * d * d * 4) == 0 and enough <= 512 * d * d * 4
                    some += apart < in_place
    assert some > 50
    assert lib.acid_linear_attention_workspace_needed(9, 1, 2, 40000, 128, 0) == 0


def test_attention_of_no_sequences_does_nothing(lib):
    assert _attend(lib, n=0, q=None, k=None, vt=None, slopes=None, o=None, ws=None, bytes=0) == 0


def _step(lib, **kw):
    a = dict(dtype=L.ACID_BF16, rows=4, heads=2, d=64, q=G, qld=384, k=G + 256, kld=384,
             v=G + 512, vld=384, slopes=2 * G, slots=3 * G, n_slots=9, sin=4 * G, sout=4 * G,
             scale=1.0, o=5 * G, old=128)
    a.update(kw)
    return lib.acid_linear_attention_step(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), BAD), (dict(rows=-1), BAD), (dict(heads=0), BAD), (dict(d=32), SHAPE),
    (dict(n_slots=-1), SHAPE), (dict(slots=None, n_slots=3), SHAPE),
    (dict(n_slots=1 << 31), SHAPE), (dict(rows=1 << 22), SHAPE), (dict(rows=65537), SHAPE),
    (dict(qld=120), SHAPE), (dict(kld=385), SHAPE), (dict(vld=1 << 33), SHAPE), (dict(old=64), SHAPE),
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(o=None), BAD),
    (dict(slopes=None), BAD), (dict(sin=None), BAD), (dict(sout=None), BAD),
    (dict(v=G + 514), BAD), (dict(sout=4 * G + 8), BAD),
    (dict(o=G + 256, old=384), BAD),          # over k's columns
    (dict(o=G + 16, old=128), BAD),           # another stride inside q
    (dict(sout=4 * G + 65536), BAD),          # part of the states read
    (dict(o=4 * G), BAD), (dict(sin=G, sout=G), BAD)])
def test_step_refusals(lib, kw, status):
    assert _step(lib, **kw) == status
    assert L.last_error()


def test_step_of_no_rows_does_nothing(lib):
    assert _step(lib, rows=0, q=None, k=None, v=None, o=None, slots=None, n_slots=0, sin=None,
                 sout=None, slopes=None) == 0


def _norm(lib, rows=10, hidden=256, **kw):
    a = L.ResidualNormArgsC()
    for key, v in dict(h=G, h_ld=256, y=2 * G, y_ld=256, h_out=G, h_out_ld=256, out=3 * G,
                       out_ld=256, y_dtype=L.ACID_BF16, out_dtype=L.ACID_BF16, post=2, pre=1,
                       res_scale=1.0, eps=1e-6).items():
        setattr(a, key, v)
    for key, v in kw.items():
        setattr(a, key, v)
    return lib.acid_residual_norm(C.byref(a), rows, hidden, None)


def test_packed_norm_arguments_are_the_structs_bytes():
    values = [*range(1, 19), 0.5, 0.25]
    assert P._NORM_ARGS.pack(*values) == bytes(L.ResidualNormArgsC(*values))


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), BAD), (dict(hidden=0), SHAPE), (dict(hidden=258), SHAPE),
    (dict(hidden=8196), SHAPE), (dict(rows=(1 << 23) + 1), SHAPE), (dict(post=3), BAD),
    (dict(pre=-1), BAD), (dict(y_dtype=5), BAD), (dict(out_dtype=5), BAD), (dict(eps=-1e-6), BAD),
    (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD),
    (dict(res_scale=float("inf")), BAD), (dict(rows_per_mod=-1), BAD), (dict(h=None), BAD),
    (dict(h_out=None), BAD), (dict(y=None, out=None), BAD), (dict(h_ld=252), SHAPE),
    (dict(y_ld=257), SHAPE), (dict(out_ld=1 << 33), SHAPE), (dict(h=G + 8), BAD),
    (dict(y=2 * G + 4), BAD), (dict(out=3 * G + 4), BAD), (dict(gate=4 * G + 4), BAD),
    (dict(h_out_ld=260), BAD),                  # h in place, but of another stride
    (dict(h_out=G + 1024), BAD),                # one row later
    (dict(out=G), BAD), (dict(out=2 * G), BAD), (dict(h_out=2 * G), BAD),
    (dict(shift=3 * G), BAD), (dict(gate=G), BAD)])
def test_norm_refusals(lib, kw, status):
    assert _norm(lib, **kw) == status
    assert L.last_error()


def test_norm_of_no_rows_does_nothing(lib):
    assert _norm(lib, rows=0, h=None, y=None, h_out=None, out=None) == 0
    assert lib.acid_residual_norm(None, 1, 256, None) == BAD


def _w4(lib, **kw):
    a = dict(xt=L.ACID_BF16, M=3, N=100, K=256, group=64, x=G, xld=256, codes=2 * G,
             scales=3 * G, bias=None, kind=L.ACID_EPI_BIAS, ot=L.ACID_F32, out=4 * G, old=100)
    a.update(kw)
    return lib.acid_linear_w4(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(xt=2), BAD), (dict(ot=-1), BAD), (dict(kind=L.ACID_EPI_QKV), UNSUPPORTED),
    (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=192), SHAPE),
    (dict(group=16), SHAPE), (dict(group=256), SHAPE), (dict(M=65537), SHAPE),
    (dict(K=1 << 23, xld=1 << 23), SHAPE), (dict(N=(1 << 22) + 1, old=1 << 23), SHAPE),
    (dict(xld=248), SHAPE), (dict(xld=257), SHAPE), (dict(old=99), SHAPE), (dict(x=None), BAD),
    (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(out=None), BAD), (dict(x=G + 8), BAD),
    (dict(codes=2 * G + 4), BAD), (dict(out=4 * G + 2), BAD), (dict(out=G), BAD),
    (dict(out=2 * G), BAD), (dict(out=3 * G), BAD), (dict(bias=4 * G), BAD)])
def test_w4_refusals(lib, kw, status):
    assert _w4(lib, **kw) == status
    assert L.last_error()


def test_w4_of_no_rows_does_nothing(lib):
    assert _w4(lib, M=0, x=None, codes=None, scales=None, out=None) == 0


@pytest.mark.parametrize("args,status", [
    ((G, 100, 256, 48, 2 * G, 3 * G), SHAPE), ((G, 100, 200, 64, 2 * G, 3 * G), SHAPE),
    ((G, 0, 256, 64, 2 * G, 3 * G), BAD), ((None, 100, 256, 64, 2 * G, 3 * G), BAD),
    ((G, 100, 256, 64, None, 3 * G), BAD), ((G, 100, 256, 64, 2 * G, None), BAD),
    ((G, 100, 256, 64, 2 * G + 8, 3 * G), BAD), ((G, 100, 256, 64, G + 1024, 3 * G), BAD),
    ((G, 100, 256, 64, 2 * G, 2 * G), BAD)])
def test_quantize_refusals(lib, args, status):
    assert lib.acid_quantize_w4(*args, None) == status
    assert L.last_error()


def test_binding_refuses_wrong_tensors():
    """Shapes, types and places are checked before the library is called."""
    t = torch.zeros
    with pytest.raises(ValueError, match="expected a tensor on"):
        P.linear_attention(t(2, 5, 64), t(2, 5, 64), t(2, 64, 8), t(2), t(5, 128))
    with pytest.raises(ValueError, match="float16"):
        P.linear_attention(t(2, 5, 64).half(), t(2, 5, 64), t(2, 64, 8), t(2), t(5, 128))
    with pytest.raises(ValueError, match="heads, L, d"):
        P.linear_attention(t(5, 64), t(5, 64), t(64, 8), t(2), t(5, 128))
    with pytest.raises(ValueError, match="n_slots"):
        P.linear_attention_step(t(1, 64), t(1, 64), t(1, 64), t(1), t(1, 64), t(64, 64))
    with pytest.raises(ValueError, match="unknown norm"):
        P.residual_norm(t(2, 8), post="batch")
    with pytest.raises(ValueError, match="without y"):
        P.residual_norm(t(2, 8), h_out=t(2, 8))
    with pytest.raises(ValueError, match="multiple of 128"):
        P.w4_shapes(16, 100)
    with pytest.raises(ValueError, match="w4_shapes"):
        P.linear_w4(t(1, 128), t(1, 64), t(1, 1, 16), t(1, 16))
    assert P.w4_shapes(17, 256, 32) == ((2, 2, 64, 16), (2, 8, 16))


class _Native:
    """The entry points as the binding calls them."""

    def __getattr__(self, name):
        return getattr(P._native()[1], name.removeprefix("acid_"))


def test_native_calls_pass_every_argument_on(lib):
    """A refusal for each argument in turn, in the same words by both ways."""
    def both(call, **kw):
        statuses = []
        for how in (lib, _Native()):
            statuses.append((call(how, **kw), L.last_error()))
        assert statuses[0] == statuses[1] and statuses[0][0] != 0, kw

    for kw in (dict(dtype=7), dict(n=-1), dict(heads=1 << 21), dict(L=-1), dict(d=80), dict(q=None), dict(k=3 * G),
               dict(k=None), dict(vt=G + 8), dict(ld=99), dict(ld=1 << 40), dict(slopes=None), dict(sin=5 * G),
               dict(sout=G), dict(o=None), dict(L=40000, ld=40000, ws=None), dict(L=40000, ld=40000, bytes=77)):
        if "bytes" in kw or "ws" in kw:
            kw.update(n=1, heads=2, d=128)
        both(_attend, **kw)
    for kw in (dict(dtype=2), dict(rows=-1), dict(rows=65537), dict(heads=0), dict(d=32), dict(q=None), dict(qld=120),
               dict(k=G + 2), dict(kld=385), dict(v=None), dict(vld=1 << 33), dict(slopes=None), dict(slots=None, n_slots=3),
               dict(n_slots=-1), dict(sin=None), dict(sout=4 * G + 8), dict(o=4 * G), dict(old=64)):
        both(_step, **kw)
    for kw in (dict(M=-1), dict(N=0), dict(K=200), dict(group=16), dict(x=None), dict(codes=2 * G + 8), dict(scales=None),
               dict(out=None)):
        both(_w4, **kw)
    native = _Native()
    a = L.ResidualNormArgsC()
    for args in ((bytes(a), -1, 256, None), (bytes(a), 4, 6, None), (None, 4, 256, None), (bytes(a), 4, 256, None)):
        assert native.acid_residual_norm(*args) == BAD or args[2] == 6
    assert native.acid_quantize_w4(G, 100, 256, 48, 2 * G, 3 * G, None) == SHAPE
    with pytest.raises(TypeError):
        native.acid_quantize_w4(G, 100, 256)
    with pytest.raises(OverflowError):
        native.acid_quantize_w4(G, 1 << 31, 256, 64, 2 * G, 3 * G, None)
    with pytest.raises(TypeError):
        native.acid_quantize_w4(G, 100.0, 256, 64, 2 * G, 3 * G, None)
