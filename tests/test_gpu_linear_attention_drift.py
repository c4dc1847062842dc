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
