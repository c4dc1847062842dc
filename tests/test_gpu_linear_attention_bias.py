"""bf16 outputs of a long prompt are off to neither side: the mean of their errors.

Inputs of one sign, so that no sum cancels and every error is relative to its output.
An output's rounding is within 2^-8 of it and of no sign in common with the others';
the mean over N of them is within 2^-8 sqrt(2 ln(2 / p) / N) but for a chance of p
(Hoeffding; p = 1e-9), as is the mean of the two-part operands' roundings, 2^-16 each of
a product.  What may be of one sign: a decay in one fp32 part over the chunks of a segment,
at most 25 here, 2^-25 each, and fp32 sums' own last bits, 2^-24 for each of the steps
(chunks) that a slope of 1 / 300 leaves of them, about 5: 2^-20 for both.
"""
import math

import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_outputs_are_off_to_neither_side(d):
    P = need_gpu()
    heads, L, C = 12, 65536, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    q, k = ((0.5 + torch.rand((heads, L, d), generator=g, device="cuda")).bfloat16() for _ in range(2))
    vt = (0.5 + torch.rand((heads, d, L), generator=g, device="cuda")).bfloat16()
    slopes = torch.full((heads,), 1 / 300, device="cuda")
    o = torch.empty((L, heads * d), dtype=torch.bfloat16, device="cuda")
    P.linear_attention(q, k, vt, slopes, o, scale=1.0)
    rate = float(slopes[0])
    i = torch.arange(C, device="cuda", dtype=torch.float64)
    weight = torch.exp(-rate * (i[:, None] - i[None, :]).clamp(min=0)) * (i[:, None] >= i[None, :])
    state = torch.zeros((heads, d, d), dtype=torch.float64, device="cuda")
    total, n = 0.0, 0
    for c in range(0, L, C):
        qc, kc = (t[:, c:c + C].double() for t in (q, k))
        vc = vt[:, :, c:c + C].double().transpose(1, 2).contiguous()
        ref = torch.matmul(torch.matmul(qc, kc.transpose(1, 2).contiguous()) * weight, vc)
        ref += torch.matmul(qc * torch.exp(-rate * (i + 1))[:, None], state)
        state = math.exp(-rate * C) * state + torch.matmul(
            (kc * torch.exp(-rate * (C - 1 - i))[:, None]).transpose(1, 2).contiguous(), vc)
        got = o[c:c + C].double().view(C, heads, d).transpose(0, 1)
        total += float((got / ref - 1).sum())
        n += ref.numel()
    bound = (2.0 ** -8 + 2.0 ** -16) * math.sqrt(2 * math.log(2e9) / n) + 2.0 ** -20
    print(f"d {d}: mean error {total / n:.3e}, bound {bound:.3e}", flush=True)
    assert abs(total / n) <= bound
