"""Exact statuses, one for each case, where test_linear_block_args accepts either of
two, and residual_norm's refusals through the native module in the same words as
through ctypes.  Nothing reaches the GPU."""
import ctypes as C

import pytest

import paper_2607_12358_amd as P
from paper_2607_12358_amd import _lib as L
from test_linear_block_args import BAD, G, SHAPE, _attend, _step, lib  # noqa: F401  (lib: fixture)


def test_a_small_workspace(lib):  # noqa: F811
    for in_place, sin in ((0, None), (1, 7 * G)):
        need = lib.acid_linear_attention_workspace_needed(L.ACID_BF16, 1, 2, 40000, 128, in_place)
        assert 0 < need <= lib.acid_linear_attention_workspace_bytes(1, 2, 40000, 128)
        for ws, size, status in ((6 * G, need - 1, SHAPE), (None, 0, SHAPE), (None, need, SHAPE), (6 * G, 0, SHAPE),
                                 (6 * G + 8, need, BAD), (5 * G, need, BAD)):
            got = _attend(lib, n=1, heads=2, L=40000, ld=40000, d=128, ws=ws, bytes=size, sin=sin, sout=sin)
            assert got == status, (ws, size, L.last_error())


def _norm_args(**kw):
    a = L.ResidualNormArgsC()
    for key, v in dict(h=G, h_ld=256, y=2 * G, y_ld=256, h_out=G, h_out_ld=256, out=3 * G, out_ld=256,
                       y_dtype=L.ACID_BF16, out_dtype=L.ACID_BF16, post=2, pre=1, res_scale=1.0, eps=1e-6, **kw).items():
        setattr(a, key, v)
    return a


@pytest.mark.parametrize("rows,hidden,kw,status", [
    (-1, 256, {}, BAD), (4, 6, {}, SHAPE), (4, 0, {}, SHAPE), (4, 8196, {}, SHAPE), ((1 << 23) + 1, 256, {}, SHAPE),
    (4, 256, None, BAD), (4, 256, dict(gate=4 * G + 4), BAD), (4, 256, dict(rows_per_mod=-1), BAD),
    (4, 256, dict(shift=3 * G), BAD), (4, 256, dict(scale=4 * G + 8), BAD), (4, 256, dict(pre_weight=G), BAD),
    (4, 256, dict(post_weight=3 * G + 512), BAD)])
def test_norm_by_both_ways(lib, rows, hidden, kw, status):  # noqa: F811
    native = P._native()[1].residual_norm
    a = None if kw is None else _norm_args(**kw)
    words = []
    for got in (lib.acid_residual_norm(None if a is None else C.byref(a), rows, hidden, None),
                native(None if a is None else bytes(a), rows, hidden, None)):
        assert got == status, L.last_error()
        words.append(L.last_error())
    assert words[0] == words[1] and words[0]


@pytest.mark.parametrize("field,value,status", [
    ("h", None, BAD), ("h", G + 8, BAD), ("h_ld", 252, SHAPE), ("y", 2 * G + 4, BAD), ("y_ld", 257, SHAPE),
    ("h_out", None, BAD), ("h_out_ld", 260, BAD), ("out", G, BAD), ("out_ld", 1 << 33, SHAPE), ("y_dtype", 5, BAD),
    ("out_dtype", -1, BAD), ("post", 3, BAD), ("pre", -1, BAD), ("res_scale", float("inf"), BAD), ("eps", float("nan"), BAD)])
def test_each_field_of_the_norms_arguments(lib, field, value, status):  # noqa: F811
    native = P._native()[1].residual_norm
    a = _norm_args()
    setattr(a, field, value)
    assert lib.acid_residual_norm(C.byref(a), 4, 256, None) == status
    words = L.last_error()
    assert native(bytes(a), 4, 256, None) == status and L.last_error() == words


def test_a_pool_of_no_slots_has_padding_rows_alone(lib):  # noqa: F811
    assert _step(lib, n_slots=0, sin=None, sout=None) == 0
    assert _step(lib, n_slots=0, sin=None, sout=None, slots=None) == SHAPE
