"""ACID_FP8_EXACT beside each epilogue: the same refusals as without it."""
import pytest

from paper_2607_12358_amd import _lib as L
from test_fp8_block_args import BAD, G, SHAPE, UNSUPPORTED, UPDATE, _linear, lib  # noqa: F401  (lib: fixture)

X = L.ACID_FP8_EXACT


@pytest.mark.parametrize("kw,status", [
    (dict(kind=L.ACID_EPI_QKV | X), UNSUPPORTED), (dict(kind=L.ACID_EPI_EULER | X), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED),
    (dict(kind=2 * X), UNSUPPORTED), (dict(kind=L.ACID_EPI_BIAS | 2 * X), UNSUPPORTED), (dict(kind=L.ACID_EPI_BIAS | X | 1 << 31 - 1), UNSUPPORTED),
    (dict(UPDATE, kind=UPDATE["kind"] | X, out_dtype=L.ACID_BF16), UNSUPPORTED), (dict(UPDATE, kind=UPDATE["kind"] | X, gate=None), BAD),
    (dict(UPDATE, kind=UPDATE["kind"] | X, residual=None), BAD), (dict(UPDATE, kind=UPDATE["kind"] | X, residual_ld=99), SHAPE),
    (dict(UPDATE, kind=UPDATE["kind"] | X, out=8 * G + 400), BAD), (dict(kind=L.ACID_EPI_BIAS_GELU | X, out=G), BAD)])
def test_refusals(lib, kw, status):  # noqa: F811
    assert _linear(lib, **kw) == status
    assert L.last_error()


def test_workspace_is_enough_for_either(lib):  # noqa: F811
    for kind in (L.ACID_EPI_BIAS, L.ACID_EPI_BIAS | X):
        need = lib.acid_linear_fp8_workspace_needed(300, 1536, 8960)
        assert need > 0
        far = dict(M=300, N=1536, K=8960, a_ld=8960, a_scales_ld=300, out_ld=1536, kind=kind, a=1 << 40, w=2 << 40, out=3 << 40)
        assert _linear(lib, **far, workspace_bytes=need - 1) == SHAPE
    assert _linear(lib, M=0, kind=L.ACID_EPI_BIAS | X, a=None, w=None, a_scales=None, w_scales=None, out=None) == 0
