"""No rows, on tensors as the shape helpers give them: nothing is done, nothing raised."""
import pytest
import torch

from fp8_util import E4M3, fp8_rows, normal, quantized_weight
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [16, 128, 144, 256, 1040])
def test_no_rows(k):
    P = need_gpu()
    n = 40
    codes, scales = fp8_rows(P, 0, k)
    assert codes.shape == (0, k) and scales.shape == (-(-k // 128), 0)
    w = quantized_weight(P, normal((k, n), k))
    v, g = torch.zeros(k, device="cuda"), torch.zeros(n, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        P.quantize_fp8(torch.zeros((0, k), device="cuda", dtype=dtype), codes, scales)
        P.linear_fp8(codes, scales, *w, torch.zeros((0, n), device="cuda", dtype=dtype), bias=g)
    P.ln_modulate_fp8(torch.zeros((0, k), device="cuda"), v, v, codes, scales)
    h = torch.zeros((0, n), device="cuda")
    P.linear_fp8(codes, scales, *w, h, gate=g, residual=h)
    # beside them, the first rows of none of a larger matrix
    some = fp8_rows(P, 5, k)
    P.quantize_fp8(normal((5, k), 1), *some)
    before = some[0].view(torch.uint8).clone(), some[1].clone()
    P.quantize_fp8(normal((5, k), 2)[:0], some[0][:0], some[1][:, :0])
    assert torch.equal(some[0].view(torch.uint8), before[0]) and torch.equal(some[1], before[1])
    assert some[0].dtype is E4M3
