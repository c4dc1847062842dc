"""The 8-bit block's calls where offsets in elements or bytes pass 2^31 and 2^32: the bits of
the same values side by side, and nothing written between them."""
import pytest
import torch

from fp8_util import E4M3, normal, quantized_rows
from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _far(shape, strides, dtype):
    """A view with these strides of a matrix that nothing fills."""
    last = sum((n - 1) * s for n, s in zip(shape, strides))
    return torch.empty(last + 1, dtype=dtype, device="cuda").as_strided(shape, strides)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rotary(dtype):
    P = need_gpu()
    tokens, heads, d, sections = 37, 2, 64, (12, 10, 10)
    rows = [normal((2 * tokens, heads * d), i, dtype=dtype) for i in range(3)]
    pos = torch.arange(3 * 2 * tokens, dtype=torch.int32, device="cuda").reshape(3, 2 * tokens)
    freqs = torch.tensor([1e4 ** (-i / 32) for i in range(32)], dtype=torch.float64, device="cuda")
    outs = [torch.zeros((2, heads, *s), dtype=dtype, device="cuda") for s in ((tokens, d), (tokens, d), (d, tokens))]
    P.rotary_qkv(*rows, pos, freqs, sections, *outs, norm="rms_row")
    # rows 2^26 apart (74 of them pass 2^32), heads 2^31, sequences 2^32
    far_rows = _far((2 * tokens, heads * d), (2 ** 26, 1), dtype)
    far_pos = _far((3, 2 * tokens), (2 ** 30 + 6, 1), torch.int32)
    far_pos.copy_(pos)
    for i in range(3):
        far_rows.copy_(rows[i])
        shape = outs[i].shape
        far = _far(shape, (2 ** 32 + 4096, 2 ** 31 + 64, 2 ** 25 + 8 if i == 2 else d, 1), dtype)
        args = [far_rows if j == i else None for j in range(3)] + [far_pos, freqs, sections]
        P.rotary_qkv(*args, *(far if j == i else None for j in range(3)), norm="rms_row")
        assert torch.equal(far, outs[i]), i
        del far


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_quantize(dtype):
    P = need_gpu()
    rows, k = 70, 144
    x = normal((rows, k), 1, dtype=dtype)
    codes, scales = quantized_rows(P, x)
    far = _far((rows, k), (2 ** 26, 1), dtype)
    far.copy_(x)
    out, s = _far((rows, k), (2 ** 26, 1), torch.uint8).view(E4M3), _far((2, 72), (2 ** 31 + 4, 1), F32)
    P.quantize_fp8(far, out, s)
    assert torch.equal(out.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s[:, :rows], scales[:, :rows])
    if dtype == F32:
        shift, scale = normal((rows, k), 2), normal((rows, k), 3)
        P.ln_modulate_fp8(x, shift, scale, codes, scales, rows_per_mod=1)
        P.ln_modulate_fp8(far, shift, scale, out, s, rows_per_mod=1)
        assert torch.equal(out.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s[:, :rows], scales[:, :rows])


def test_weight_and_products():
    """4.3e9 codes: blocks at either side of 2^31 and 2^32, and the last."""
    P = need_gpu()
    n, k = 2 ** 18 + 136, 2 ** 14 + 16
    shape, sshape = P.fp8_weight_shapes(n, k)
    codes = torch.empty(shape, dtype=torch.uint8, device="cuda")
    scales = torch.empty(sshape, device="cuda")
    w = torch.zeros((k, n), device="cuda")
    starts = [2 ** 31 // k // 128 * 128, 2 ** 32 // k // 128 * 128, n - 136]
    for i, at in enumerate(starts):
        w[:, at:at + 136] = normal((k, 136), 10 + i)
    P.quantize_fp8_weight(w, codes.view(E4M3), scales)
    for at in starts:
        part = torch.empty((136, k), dtype=torch.uint8, device="cuda")
        s = torch.empty((2, sshape[1]), device="cuda")
        P.quantize_fp8_weight(w[:, at:at + 136].contiguous(), part.view(E4M3), s)
        assert torch.equal(codes[at:at + 136], part), at
        assert torch.equal(scales[at // 128:at // 128 + 2], s), at
    del w
    # whole numbers, whose sums are exact in any order
    scales.fill_(1.0)
    codes.zero_()
    small = torch.tensor([-2.0, -1.0, 0.0, 1.0, 2.0], device="cuda").to(E4M3).view(torch.uint8)
    for i, at in enumerate(starts):
        codes[at:at + 136] = small[torch.randint(0, 5, (136, k), device="cuda", generator=torch.Generator("cuda").manual_seed(i))]
    for m in (1, 13, 300):
        a = small[torch.randint(0, 5, (m, k), device="cuda", generator=torch.Generator("cuda").manual_seed(m))].view(E4M3)
        sa = torch.ones((sshape[1], (m + 3) // 4 * 4), device="cuda")
        for dtype in (F32, BF16):
            out = torch.empty((m, n), dtype=dtype, device="cuda")
            P.linear_fp8(a, sa, codes.view(E4M3), scales, out)
            want = torch.zeros((m, n), device="cuda")
            for at in starts:
                want[:, at:at + 136] = a.float() @ codes[at:at + 136].view(E4M3).float().t()
            assert torch.equal(out, want.to(dtype)), (m, dtype)
