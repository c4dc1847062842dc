"""One linear-attention block as it would be used: a prompt through the fused
GEMM, chunked attention and the seam, then tokens through 4-bit products,
single-token attention and the seam, against the same block in 64 bits."""
import numpy as np
import pytest
import torch

from gpu_util import assert_close_to_scale, need_gpu
from oracle import linear_block as B

pytestmark = pytest.mark.gpu
HEADS, D, H, G = 4, 64, 256, 64


def _f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_then_tokens(dtype):
    P = need_gpu()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    L, T = 150, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(3)

    def rnd(*s, std=1.0, m=0.0):
        return std * torch.randn(s, generator=g, device="cuda") + m

    def w4(n, k):  # the same weights in both forms: 4-bit, and their values for the GEMM
        w = rnd(k, n, std=0.05)
        cs, ss = P.w4_shapes(n, k, G)
        codes, scales = torch.empty(cs, dtype=torch.uint8, device="cuda"), torch.empty(ss, device="cuda")
        P.quantize_w4(w, codes, scales)
        full = B.w4_weights(codes.cpu().numpy(), scales.cpu().numpy(), n)
        return codes, scales, torch.from_numpy(full).cuda().to(dt).contiguous(), full

    qkv, proj = w4(3 * H, H), w4(H, H)
    b_qkv, b_o = rnd(3 * H, std=0.1), rnd(H, std=0.1)
    slopes = torch.tensor([0.0, 0.01, 0.1, 1.0], device="cuda")
    gate, shift, scale, shift2, scale2 = (rnd(H, std=0.3) for _ in range(5))
    post_w = rnd(H, std=0.1, m=1.0)
    seam = dict(post="rms", post_weight=post_w, gate=gate, pre="layer", shift=shift2, scale=scale2)

    x = rnd(L + T, H)
    h = x.clone()
    a = torch.empty((L + T, H), dtype=dt, device="cuda")
    P.residual_norm(h, out=a, shift=shift, scale=scale)          # the first norm, no block before it
    # prompt
    q, k = (torch.empty((HEADS, L, D), dtype=dt, device="cuda") for _ in range(2))
    vt = torch.empty((HEADS, D, (L + 7) // 8 * 8), dtype=dt, device="cuda")
    P.linear(a[:L], qkv[2], P.ACID_EPI_QKV, b_qkv, q=q, k=k, vt=vt, n_heads=HEADS, head_dim=D)
    o = torch.empty((L, H), dtype=dt, device="cuda")
    state = torch.empty((HEADS, D, D), device="cuda")
    P.linear_attention(q, k, vt, slopes, o, state_out=state)
    y = torch.empty((L, H), device="cuda")
    P.linear(o, proj[2], P.ACID_EPI_BIAS, b_o, out=y)
    nxt = torch.empty((L + T, H), dtype=dt, device="cuda")
    P.residual_norm(h[:L], y, out=nxt[:L], **seam)
    # tokens, one at a time on the prompt's state
    pool = torch.zeros((3, HEADS, D, D), device="cuda")
    pool[2] = state
    slot = torch.tensor([2], dtype=torch.int32, device="cuda")
    for t in range(L, L + T):
        row = torch.empty((1, 3 * H), dtype=dt, device="cuda")
        P.linear_w4(a[t:t + 1], qkv[0], qkv[1], row, bias=b_qkv)
        o1 = torch.empty((1, H), dtype=dt, device="cuda")
        P.linear_attention_step(row[:, :H], row[:, H:2 * H], row[:, 2 * H:], slopes, o1, pool,
                                slots=slot)
        y1 = torch.empty((1, H), device="cuda")
        P.linear_w4(o1, proj[0], proj[1], y1, bias=b_o)
        P.residual_norm(h[t:t + 1], y1, out=nxt[t:t + 1], **seam)
    # 64 bits
    _, a_ref = B.residual_norm(_f64(x), shift=_f64(shift), scale=_f64(scale))
    r = a_ref @ qkv[3].T + _f64(b_qkv)
    heads = [r[:, i * H:(i + 1) * H].reshape(L + T, HEADS, D).transpose(1, 0, 2) for i in range(3)]
    o_ref, s_ref = B.linear_attention(*heads, _f64(slopes), scale=D ** -0.5)
    h_ref, n_ref = B.residual_norm(_f64(x), o_ref @ proj[3].T + _f64(b_o),
                                   **{k: _f64(v) if torch.is_tensor(v) else v for k, v in seam.items()})
    bf16 = dtype == "bf16"
    assert_close_to_scale(_f64(h), h_ref, bf16, "residual stream")
    assert_close_to_scale(_f64(nxt), n_ref, bf16, "next input")
    assert_close_to_scale(_f64(pool[2]), s_ref, bf16, "state")
    assert (pool[:2] == 0).all()
