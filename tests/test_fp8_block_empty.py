"""No rows: the 8-bit block's calls have nothing to do, whatever stride an empty matrix of scales has
(torch's of [groups, 0] is 1)."""
import ctypes as C

import pytest

from paper_2607_12358_amd import _lib as L


@pytest.mark.parametrize("K", [16, 128, 144, 256, 1040])
@pytest.mark.parametrize("ld", [0, 1, 3, 4])
def test_strides_of_no_scales(K, ld):
    lib = L.lib()
    for dtype in (L.ACID_BF16, L.ACID_F32):
        assert lib.acid_quantize_fp8(dtype, 0, K, None, K, None, K, None, ld, None) == 0
    assert lib.acid_ln_modulate_fp8(0, K, None, K, None, None, 0, None, K, None, ld, None) == 0
    for kind, dtype in ((L.ACID_EPI_BIAS, L.ACID_BF16), (L.ACID_EPI_BIAS_GELU, L.ACID_F32), (L.ACID_EPI_GATE_RESIDUAL, L.ACID_F32)):
        a = L.LinearFp8ArgsC(a_ld=K, a_scales_ld=ld, residual_ld=40, out_ld=40, kind=kind, out_dtype=dtype)
        assert lib.acid_linear_fp8(C.byref(a), 0, 40, K, None) == 0
