"""Refusals of the linear-attention block's calls that need tensors on the device:
each is the framework's own error, and nothing is launched."""
import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


def z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def test_heads_of_nothing():
    P = need_gpu()
    with pytest.raises(P.AcidError, match="head_dim 0"):
        P.linear_attention(z(2, 5, 0), z(2, 5, 0), z(2, 0, 8), z(2), z(5, 0))
    with pytest.raises(P.AcidError, match="head_dim 0"):
        P.linear_attention_step(z(1, 0), z(1, 0), z(1, 0), z(2), z(1, 0), z(1, 2, 0, 0))
    with pytest.raises(P.AcidError, match="n_heads"):
        P.linear_attention(z(0, 5, 64), z(0, 5, 64), z(0, 64, 8), z(0), z(5, 0))


def test_rows_of_other_axes():
    P = need_gpu()
    for q in (torch.tensor(1.0, device="cuda"), z(64), z(1, 1, 64)):
        with pytest.raises(ValueError, match="q: expected"):
            P.linear_attention_step(q, z(1, 64), z(1, 64), z(1), z(1, 64), z(1, 1, 64, 64))
