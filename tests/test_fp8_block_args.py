"""Argument checks of the 8-bit block's entry points: every call here is refused, or
has nothing to do, before any GPU work (made-up addresses are never looked at)."""
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


def _rows(lib, **kw):
    a = dict(dtype=L.ACID_BF16, rows=10, K=256, x=G, xld=256, codes=2 * G, cld=256, scales=3 * G, sld=12)
    a.update(kw)
    return lib.acid_quantize_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), BAD), (dict(rows=-1), BAD), (dict(K=0), BAD), (dict(K=250), SHAPE), (dict(K=1 << 23, xld=1 << 23, cld=1 << 23), SHAPE),
    (dict(rows=1 << 31, sld=1 << 31), SHAPE), (dict(rows=1 << 31, K=16, sld=1 << 31), SHAPE), (dict(xld=255), SHAPE), (dict(xld=260), SHAPE), (dict(xld=1 << 33), SHAPE),
    (dict(dtype=L.ACID_F32, xld=258), SHAPE), (dict(cld=240), SHAPE), (dict(cld=264), SHAPE), (dict(sld=8), SHAPE), (dict(sld=13), SHAPE),
    (dict(x=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(x=G + 8), BAD), (dict(codes=2 * G + 8), BAD),
    (dict(scales=3 * G + 4), BAD), (dict(codes=G), BAD), (dict(scales=G + 512), BAD), (dict(scales=2 * G + 256), BAD)])
def test_rows_refusals(lib, kw, status):
    assert _rows(lib, **kw) == status
    assert L.last_error()


def _norm(lib, **kw):
    a = dict(rows=10, hidden=256, x=G, xld=256, shift=4 * G, scale=5 * G, per=3, codes=2 * G, cld=256, scales=3 * G, sld=12)
    a.update(kw)
    return lib.acid_ln_modulate_fp8(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), BAD), (dict(hidden=0), BAD), (dict(hidden=264), SHAPE), (dict(hidden=8208, xld=8208, cld=8208), SHAPE),
    (dict(rows=(1 << 23) + 1, sld=(1 << 23) + 4), SHAPE), (dict(xld=254), SHAPE), (dict(xld=258), SHAPE), (dict(per=-1), BAD),
    (dict(x=None), BAD), (dict(shift=None), BAD), (dict(scale=None), BAD), (dict(codes=None), BAD), (dict(scales=None), BAD),
    (dict(shift=4 * G + 4), BAD), (dict(codes=4 * G), BAD), (dict(scales=5 * G + 1024), BAD), (dict(codes=G + 1024), BAD)])
def test_norm_refusals(lib, kw, status):
    assert _norm(lib, **kw) == status
    assert L.last_error()


def _weight(lib, **kw):
    a = dict(w=G, N=100, K=256, codes=2 * G, scales=3 * G)
    a.update(kw)
    return lib.acid_quantize_fp8_weight(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=100), SHAPE), (dict(N=(1 << 22) + 1), SHAPE), (dict(K=1 << 23), SHAPE), (dict(w=None), BAD),
    (dict(codes=None), BAD), (dict(scales=None), BAD), (dict(codes=2 * G + 8), BAD), (dict(w=G + 2), BAD), (dict(codes=G), BAD),
    (dict(scales=G + 1024), BAD), (dict(scales=2 * G + 1024), BAD)])
def test_weight_refusals(lib, kw, status):
    assert _weight(lib, **kw) == status
    assert L.last_error()


def test_rows_of_nothing_do_nothing(lib):
    assert _rows(lib, rows=0, x=None, codes=None, scales=None, sld=0) == 0
    assert _norm(lib, rows=0, x=None, shift=None, scale=None, codes=None, scales=None, sld=0) == 0


def _linear(lib, M=10, N=100, K=256, **kw):
    a = L.LinearFp8ArgsC()
    for key, v in dict(a=G, a_ld=256, a_scales=2 * G, a_scales_ld=12, w=3 * G, w_scales=4 * G, bias=5 * G, out=6 * G, out_ld=100,
                       kind=L.ACID_EPI_BIAS, out_dtype=L.ACID_BF16, workspace=10 * G, workspace_bytes=1 << 29).items():
        setattr(a, key, v)
    for key, v in kw.items():
        setattr(a, key, v)
    return lib.acid_linear_fp8(C.byref(a), M, N, K, None)


UPDATE = dict(kind=L.ACID_EPI_GATE_RESIDUAL, out_dtype=L.ACID_F32, gate=7 * G, residual=8 * G, residual_ld=100)


@pytest.mark.parametrize("kw,status", [
    (dict(out_dtype=3), BAD), (dict(kind=L.ACID_EPI_QKV), UNSUPPORTED), (dict(kind=L.ACID_EPI_EULER), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED),
    (dict(UPDATE, out_dtype=L.ACID_BF16), UNSUPPORTED), (dict(M=-1), BAD), (dict(N=0), BAD), (dict(K=0), BAD), (dict(K=250), SHAPE),
    (dict(K=1 << 23, a_ld=1 << 23), SHAPE), (dict(N=(1 << 22) + 1, out_ld=1 << 23), SHAPE), (dict(M=(1 << 24) + 1, a_scales_ld=1 << 25), SHAPE),
    (dict(a_ld=240), SHAPE), (dict(a_ld=264), SHAPE), (dict(a_ld=1 << 24), SHAPE), (dict(out_ld=99), SHAPE), (dict(out_ld=1 << 33), SHAPE),
    (dict(UPDATE, residual_ld=99), SHAPE), (dict(a_scales_ld=8), SHAPE), (dict(a_scales_ld=14), SHAPE),
    (dict(a=None), BAD), (dict(w=None), BAD), (dict(a_scales=None), BAD), (dict(w_scales=None), BAD), (dict(out=None), BAD),
    (dict(UPDATE, gate=None), BAD), (dict(UPDATE, residual=None), BAD), (dict(a=G + 8), BAD), (dict(w=3 * G + 8), BAD),
    (dict(a_scales=2 * G + 4), BAD), (dict(out=6 * G + 1), BAD), (dict(bias=5 * G + 2), BAD), (dict(UPDATE, gate=7 * G + 2), BAD),
    (dict(out=G), BAD), (dict(out=2 * G), BAD), (dict(out=3 * G + 200), BAD), (dict(out=4 * G), BAD), (dict(out=5 * G + 100), BAD),
    (dict(UPDATE, out=7 * G), BAD), (dict(UPDATE, out=8 * G + 400), BAD), (dict(UPDATE, out=8 * G, out_ld=104), BAD)])
def test_linear_refusals(lib, kw, status):
    assert _linear(lib, **kw) == status
    assert L.last_error()


def test_linear_of_no_rows_does_nothing(lib):
    assert _linear(lib, M=0, a=None, w=None, a_scales=None, w_scales=None, out=None, workspace=None, workspace_bytes=0) == 0
    assert lib.acid_linear_fp8(None, 1, 16, 16, None) == BAD


def test_linear_workspace(lib):
    some = 0
    for M in (1, 5, 16, 17, 64, 100, 256, 300, 1000, 32760):
        for N in (1, 100, 1536, 8960):
            for K in (16, 400, 1536, 8960, 1 << 20):
                need = lib.acid_linear_fp8_workspace_needed(M, N, K)
                assert need % 16 == 0 and need < 1 << 30
                if need:
                    some += 1
                    kw = dict(M=M, N=N, K=K, a_ld=K, a_scales_ld=(M + 3) // 4 * 4, out_ld=N)
                    far = dict(a=1 << 40, w=2 << 40, out=3 << 40)
                    assert _linear(lib, **kw, **far, workspace_bytes=need - 1) == SHAPE
                    assert _linear(lib, **kw, **far, workspace=None, workspace_bytes=need) == BAD
                    assert _linear(lib, **kw, **far, workspace=10 * G + 8, workspace_bytes=need) == BAD
                    assert _linear(lib, **kw, **far, workspace=(3 << 40), workspace_bytes=need) == BAD
                    assert _linear(lib, **kw, **far, workspace=(2 << 40), workspace_bytes=need) == BAD
    for bad in ((0, 16, 16), (-1, 16, 16), (4, 0, 16), (4, 16, 0), (4, 16, 24), (1 << 40, 16, 16), (4, 1 << 30, 16)):
        assert lib.acid_linear_fp8_workspace_needed(*bad) == 0


def _heads(lib, n_seq=1, tokens=10, **kw):
    a = L.RotaryQkvArgsC()
    for key, v in dict(q=G, k=G + 512, v=G + 768, q_ld=512, k_ld=512, v_ld=512, q_out=2 * G, k_out=3 * G, vt=4 * G, q_head=640, q_row=64,
                       q_seq=0, k_head=640, k_row=64, k_seq=0, vt_head=64 * 16, vt_row=16, vt_seq=0, positions=5 * G, positions_ld=10,
                       freqs=6 * G, in_dtype=L.ACID_BF16, out_dtype=L.ACID_BF16, heads=4, kv_heads=2, head_dim=64, axes=3, pairing=0,
                       norm=0, q_scale=1.0, eps=1e-6).items():
        setattr(a, key, v)
    a.sections[:] = kw.pop("sections", [8, 12, 12, 0])
    for key, v in kw.items():
        setattr(a, key, v)
    return lib.acid_rotary_qkv(C.byref(a), n_seq, tokens, None)


@pytest.mark.parametrize("kw,status", [
    (dict(in_dtype=2), BAD), (dict(out_dtype=-1), BAD), (dict(norm=4), BAD), (dict(norm=-1), BAD), (dict(pairing=2), BAD),
    (dict(positions_f32=2), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(q_scale=float("inf")), BAD),
    (dict(n_seq=-1), BAD), (dict(tokens=-1), BAD), (dict(q=None), BAD), (dict(q_out=None), BAD), (dict(k=None), BAD), (dict(vt=None), BAD),
    (dict(head_dim=96), SHAPE), (dict(heads=0), SHAPE), (dict(heads=1025), SHAPE), (dict(kv_heads=0), SHAPE), (dict(axes=0), SHAPE),
    (dict(axes=5), SHAPE), (dict(sections=[8, -1, 12, 0]), SHAPE), (dict(sections=[12, 12, 12, 0]), SHAPE),
    (dict(sections=[33, 0, 0, 0]), SHAPE), (dict(sections=[8, 12, 11, 0], pairing=1), SHAPE), (dict(q_ld=248), SHAPE), (dict(q_ld=516), SHAPE),
    (dict(k_ld=127), SHAPE), (dict(v_ld=1 << 33), SHAPE), (dict(tokens=1 << 31), SHAPE), (dict(n_seq=1 << 21, tokens=1), SHAPE),
    (dict(q_row=60), SHAPE), (dict(q_row=68, q_head=680), SHAPE), (dict(q_head=639), SHAPE), (dict(q_head=0), SHAPE), (dict(q_row=-64), SHAPE),
    (dict(k_head=1 << 41), SHAPE), (dict(vt_row=9), SHAPE), (dict(vt_head=1000), SHAPE),
    (dict(n_seq=2, tokens=5, q_seq=1000), SHAPE), (dict(n_seq=2, tokens=5, q_seq=2564), SHAPE), (dict(positions=None), BAD), (dict(freqs=None), BAD), (dict(positions_ld=9), SHAPE),
    (dict(q_weight=7 * G), BAD), (dict(q_bias=7 * G, norm=2), BAD), (dict(k_bias=7 * G, norm=3), BAD), (dict(q=G + 8), BAD),
    (dict(q_out=2 * G + 8), BAD), (dict(vt=4 * G + 1), BAD), (dict(freqs=6 * G + 4), BAD), (dict(positions=5 * G + 2), BAD),
    (dict(norm=2, q_weight=7 * G + 4), BAD), (dict(q_out=G), BAD), (dict(q_out=G, q_head=64, q_row=512, out_dtype=L.ACID_F32), BAD),
    (dict(q_out=G + 512, q_head=64, q_row=512), BAD), (dict(k_out=G, k_head=64, k_row=512), BAD), (dict(k_out=2 * G + 1280), BAD),
    (dict(vt=3 * G + 64), BAD), (dict(vt=5 * G), BAD), (dict(k_out=6 * G), BAD), (dict(norm=3, k_weight=2 * G + 16), BAD),
    (dict(n_seq=1 << 19, tokens=64, positions_ld=1 << 25, q_seq=1 << 20, k_seq=1 << 20, vt_seq=1 << 20, q_head=4096, k_head=4096, vt_row=64, vt_head=4096, q=1 << 50, k=2 << 50, v=3 << 50, q_out=4 << 50,
          k_out=5 << 50, vt=6 << 50, positions=7 << 50, kv_heads=32, heads=32, q_ld=2048, k_ld=2048, v_ld=2048), SHAPE)])
def test_heads_refusals(lib, kw, status):
    assert _heads(lib, **kw) == status
    assert L.last_error()


def test_heads_of_nothing_do_nothing(lib):
    assert _heads(lib, tokens=0, positions=None, freqs=None) == 0
    assert _heads(lib, n_seq=0) == 0
    assert _heads(lib, q=None, k=None, v=None, q_out=None, k_out=None, vt=None) == 0
    assert lib.acid_rotary_qkv(None, 1, 1, None) == BAD


def test_packed_arguments_are_the_structs_bytes():
    a = [*range(1, 17)]
    assert P._FP8_ARGS.pack(*a) == bytes(L.LinearFp8ArgsC(*a))
    names = [n for n, _ in L.RotaryQkvArgsC._fields_]
    values = dict(zip(names, range(1, len(names) + 1)))
    values["sections"] = (C.c_int32 * 4)(91, 92, 93, 94)
    values["q_scale"], values["eps"] = 0.5, 0.25
    flat = [x for n in names for x in (values[n] if n == "sections" else [values[n]])]
    assert P._ROTARY_ARGS.pack(*flat) == bytes(L.RotaryQkvArgsC(*(values[n] for n in names)))


def test_shapes():
    assert P.fp8_shapes(5, 144) == ((5, 144), (2, 8)) and P.fp8_shapes(0, 16) == ((0, 16), (1, 0))
    assert P.fp8_weight_shapes(129, 144) == ((129, 144), (2, 2))
    for f, a in ((P.fp8_shapes, (-1, 16)), (P.fp8_shapes, (1, 24)), (P.fp8_weight_shapes, (0, 16)), (P.fp8_weight_shapes, (1, 8))):
        with pytest.raises(ValueError):
            f(*a)


def test_tensors_of_the_cpu_are_refused():
    x, e = torch.zeros(4, 32), torch.zeros(4, 32).to(torch.float8_e4m3fn)
    for call in (lambda: P.quantize_fp8(x, e, torch.zeros(1, 4)), lambda: P.quantize_fp8_weight(x, e, torch.zeros(1, 1)),
                 lambda: P.ln_modulate_fp8(x, x[0], x[0], e, torch.zeros(1, 4)), lambda: P.linear_fp8(e, torch.zeros(1, 4), e, torch.zeros(1, 1), x),
                 lambda: P.rotary_qkv(torch.zeros(4, 64), None, None, torch.zeros(1, 4), torch.zeros(8), (8,), torch.zeros(1, 4, 64), None, None)):
        with pytest.raises(ValueError, match="GPU"):
            call()
