"""A state's decay over thousands of tokens and calls: a factor that is rounded
to fp32 is off to the same side each time, which adds up.

Bounds.  With u = 2^-24, N decays of a state that grows or fades slowly (slopes below
1 / N) round each of its values N times, to nearest, so a value is within (N + 4) u
of itself, and the roundings of values that differ in all their bits have no
common sign.  The mean over E of them is then within (N + 4) u sqrt(2 ln(2 / p) / E)
but for a chance of p (Hoeffding); p = 1e-9 and E = 16384 make that 0.0512 (N + 4) u.
A factor off by f u moves that mean by f N u where the state only fades, and by half
of that where it grows from nothing: f is 0.36, 0.36 and 0.46 for the first three
slopes below.
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import need_gpu

pytestmark = pytest.mark.gpu
D = 128
SLOPES = (1e-4, 7e-5, 2e-5, 0.0)
U = 2.0 ** -24


def _inputs(fading, seed, heads=len(SLOPES)):
    """k, v fp32 [heads, D] and a state, all of one sign; the state alone
    (k = 0), or k and v alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (0.5 + torch.rand((heads, D), generator=g, device="cuda") for _ in range(2))
    state = 0.5 + torch.rand((heads, D, D), generator=g, device="cuda")
    return (torch.zeros_like(k), v, state) if fading else (k, v, torch.zeros_like(state))


def _check(got, k, v, state, tokens, decays, what):
    """got: the state after `tokens` tokens of the same k and v."""
    k, v, state, got = (t.double().cpu().numpy() for t in (k, v, state, got))
    for h, slope in enumerate(SLOPES):
        slope = float(np.float32(slope))
        sums = -math.expm1(-slope * tokens) / -math.expm1(-slope) if slope else tokens
        want = math.exp(-slope * tokens) * state[h] + sums * k[h][:, None] * v[h][None, :]
        off = (got[h] - want) / want
        bound = (decays + 4) * U
        mean = math.sqrt(2 * math.log(2e9) / off.size) * bound
        print(f"{what} slope {slope:.1e}: mean / bound {off.mean() / mean:.3f}, "
              f"worst / bound {np.abs(off).max() / bound:.3f}", flush=True)
        assert np.abs(off).max() <= bound, (what, slope)
        assert abs(off.mean()) <= mean, (what, slope)


@pytest.mark.parametrize("fading", [True, False])
def test_tokens_one_by_one(fading):
    """8192 tokens of one slot."""
    P = need_gpu()
    n = 8192
    k, v, state = _inputs(fading, 1)
    rows = [t.reshape(1, -1).expand(n, -1).contiguous() for t in (k, v)]
    pool, o = state[None].clone(), torch.empty((n, len(SLOPES) * D), device="cuda")
    P.linear_attention_step(rows[0], rows[0], rows[1], torch.tensor(SLOPES, device="cuda"), o, pool,
                            slots=torch.zeros(n, dtype=torch.int32, device="cuda"))
    _check(pool[0], k, v, state, n, n, f"steps, {'fading' if fading else 'growing'}")


# (dtype, tokens a call, head_dim, in place, roundings of a fading state's value a call): one chunk or
# two, segments whose states the outputs' kernel adds, segments that are scanned, segments that
# each make their own state
STREAMS = [("bf16", 1, 64, True, 1), ("f32", 1, 128, True, 1), ("bf16", 17, 128, True, 1), ("f32", 40, 64, True, 1),
           ("bf16", 65, 64, True, 2), ("f32", 300, 64, True, 3), ("f32", 700, 128, True, 3),
           ("bf16", 700, 64, True, 3), ("bf16", 300, 64, False, 4)]


@pytest.mark.parametrize("dtype,L,d,in_place,roundings", STREAMS)
def test_stream_of_prompts(dtype, L, d, in_place, roundings):
    """400 calls of L tokens with k = 0, each from the state before; slopes for
    which exp(-slope L) lies far from the fp32 values beside it."""
    P = need_gpu()
    calls, each = 400, 4
    slopes = []
    for i in range(1000):
        slope = float(np.float32(1e-4 + 1e-7 * i))
        f = (float(np.float32(math.exp(-slope * L))) / math.exp(-slope * L) - 1) / U
        if abs(f) > 0.42 and len(slopes) < 3:
            slopes.append(slope)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    heads = each * len(slopes)
    g = torch.Generator(device="cuda")
    g.manual_seed(L)
    state = 0.5 + torch.rand((heads, d, d), generator=g, device="cuda")
    q, k = (torch.zeros((heads, L, d), dtype=dt, device="cuda") for _ in range(2))
    vt = torch.ones((heads, d, (L + 7) // 8 * 8), dtype=dt, device="cuda")
    sl = torch.tensor(np.repeat(slopes, each), dtype=torch.float32, device="cuda")
    o = torch.empty((L, heads * d), dtype=dt, device="cuda")
    now, then = state.clone(), torch.empty_like(state)
    for _ in range(calls):
        if in_place:
            P.linear_attention(q, k, vt, sl, o, state_in=now, state_out=now)
        else:
            P.linear_attention(q, k, vt, sl, o, state_in=now, state_out=then)
            now, then = then, now
    for i, slope in enumerate(slopes):
        part = slice(i * each, (i + 1) * each)
        want = math.exp(-slope * L * calls) * state[part].double().cpu().numpy()
        off = now[part].double().cpu().numpy() / want - 1
        bound = (roundings * calls + 4) * U
        mean = math.sqrt(2 * math.log(2e9) / off.size) * bound
        print(f"{dtype} {L} tokens, slope {slope:.3e}: mean / bound {off.mean() / mean:.3f}, "
              f"worst / bound {np.abs(off).max() / bound:.3f}", flush=True)
        assert np.abs(off).max() <= bound and abs(off.mean()) <= mean, slope
