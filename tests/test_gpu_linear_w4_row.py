"""One row through linear_w4: the shapes on both sides of the forms it is read
in, with the bounds that test_gpu_linear_w4 derives, and the same bits as that row
among others where the sums are added in the same order."""
import pytest
import torch

from gpu_util import need_gpu
from test_gpu_linear_w4 import DT, _check, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k", [(1, 128), (16, 128), (17, 384), (300, 1024), (4080, 2048), (4096, 4096), (4097, 4096),
                                 (4112, 1152), (1536, 8960), (2048, 28672)])
@pytest.mark.parametrize("group", [32, 128])
def test_sizes(n, k, group):
    P = need_gpu()
    for xt, ot in (("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")):
        _check(P, 1, n, k, group, xt, ot, seed=3)
    _check(P, 1, n, k, group, "bf16", "bf16", gelu=True, x_pad=8, out_pad=3, seed=4)


@pytest.mark.parametrize("n,k", [(40, 256), (4096, 1536), (1536, 8960)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_a_row_is_the_same_alone_and_among_others(n, k, group):
    """The waves take the same blocks and their sums are added in one order, so a
    row's bits do not depend on how it is read."""
    P = need_gpu()
    _, codes, scales = _weights(P, n, k, group)
    x = torch.randn((3, k), device="cuda").bfloat16()
    for ot in DT.values():
        three, one = torch.empty((3, n), device="cuda", dtype=ot), torch.empty((1, n), device="cuda", dtype=ot)
        P.linear_w4(x, codes, scales, three)
        for r in range(3):
            P.linear_w4(x[r:r + 1], codes, scales, one)
            assert torch.equal(one[0], three[r]), r
