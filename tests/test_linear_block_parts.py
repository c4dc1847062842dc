"""Each part of a value that goes into its product as several bf16 ones.

Inputs on which nothing is left to hide a part behind: every sum has one term, so the
bounds are a few fp32 steps of the result itself.

linear_w4, one input of a row, or one in each group: a part times 16 + c, and times 24,
is exact (8 bits times 5), and so is their difference.  Roundings: the scale onto each of
the three parts, an addition for each of a wave's groups that has an input, for each of
at most 16 waves, for the three parts: with A the sum of the terms' sizes, (inputs + 24)
2^-24 A.  One part lost is up to 2^-8 (the second) or 2^-16 (the third) of its term.

linear_attention's state, one token of a head with k: S = exp(-slope n) k v.  The token's
decay within its segment (two exp2 and their product, with arguments below 1: 8 steps), its
product with v, three parts added, and one rounding for each chunk, and each form of adding
segments up, after it: (chunks + 24) 2^-24 of the value.  The third part lost is up to 2^-16.
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import assert_elementwise, need_gpu
from oracle import linear_block as B

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _cut(x):
    """fp32 values cut to their first eight significant bits."""
    return (np.asarray(x, np.float32).view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)


def _parts(x, n):
    """The sum of the first n of the parts that fp32 values are cut into."""
    total, rest = np.zeros(x.shape), np.asarray(x, np.float32)
    for _ in range(n):
        p = _cut(rest)
        total, rest = total + p, rest - p
    return total


def _sparse_rows(m, k, group, seed, single=False):
    """fp32 rows with one input, or one in each group, of full significands."""
    rng = np.random.default_rng(seed)
    x = np.zeros((m, k), np.float32)
    for r in range(m):
        at = np.arange(0, k, group) + rng.integers(0, group, k // group)
        at = at[r % len(at):][:1] if single else at
        x[r, at] = rng.standard_normal(len(at))
    return x


def _w4_bound(x, codes, scales, n):
    """(reference, bound)"""
    inputs = int((x != 0).sum(1).max())
    w = B.w4_weights(codes, scales, n)
    return x.astype(np.float64) @ w.T, (inputs + 24) * U * (np.abs(x.astype(np.float64)) @ np.abs(w).T)


def _w4(n, k, group, seed):
    rng = np.random.default_rng(seed)
    w = (0.02 * rng.standard_normal((k, n))).astype(np.float32)
    return B.w4_pack(*B.w4_quantize(w, group))


@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_a_lost_part_of_x_exceeds_the_bound(group, single):
    x = _sparse_rows(7, 1152, group, 0, single)
    codes, scales = _w4(50, 1152, group, 1)
    ref, bound = _w4_bound(x, codes, scales, 50)
    for parts in (3, 2, 1):
        over = np.abs(B.linear_w4(_parts(x, parts), codes, scales, 50) - ref) > bound
        assert over.any() == (parts < 3), (parts, over.mean())
        if single:  # most rows lose something in every output whose weight is not zero
            assert parts == 3 or np.median(over.mean(1)) > 0.5, (parts, over.mean(1))


@pytest.mark.gpu
@pytest.mark.parametrize("single", [False, True])
@pytest.mark.parametrize("m", [1, 3, 7, 23])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(50, 1152), (7000, 256), (14400, 640)])
def test_w4_rows_keep_every_bit(m, group, n, k, single):
    P = need_gpu()
    x = _sparse_rows(m, k, group, m, single)
    codes, scales = _w4(n, k, group, 2)
    ref, bound = _w4_bound(x, codes, scales, n)
    out = torch.full((m, n), 7.0, device="cuda")
    dev = [torch.from_numpy(t).cuda() for t in (x, codes, scales)]
    P.linear_w4(*dev, out)
    assert_elementwise(out.double().cpu().numpy(), ref, bound + 1e-40, 0.0, f"{m}x{n}x{k} g{group}")


def _state(k, v, slopes, at, L):
    """fp64 [heads, d, d]: one token of each head."""
    fade = np.exp(-slopes.astype(np.float64) * (L - 1 - np.asarray(at)))
    return fade[:, None, None] * k.astype(np.float64)[:, :, None] * v.astype(np.float64)[:, None, :]


def _bf16(rng, *shape):
    return _cut(rng.standard_normal(shape).astype(np.float32))


def test_a_lost_part_of_v_exceeds_the_bound():
    rng = np.random.default_rng(3)
    slopes, at, L = np.full(4, 1e-3, np.float32), [3, 70, 400, 699], 700
    k, v = _bf16(rng, 4, 64), _bf16(rng, 4, 64)
    ref = _state(k, v, slopes, at, L)
    faded = (np.exp(-slopes.astype(np.float64) * (L - 1 - np.asarray(at)))[:, None] * v).astype(np.float32)
    for parts, least in ((3, 0.0), (2, 0.4)):
        got = k.astype(np.float64)[:, :, None] * _parts(faded, parts)[:, None, :]
        over = np.abs(got - ref)[:3] > (11 + 24) * U * np.abs(ref)[:3]  # (the last token has no decay)
        assert over.mean() >= least and (parts < 3 or not over.any()), (parts, over.mean())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("heads,L,d", [(8, 40, 64), (8, 64, 128), (8, 200, 64), (8, 700, 128), (64, 500, 64), (20, 1000, 128),
                                       (150, 300, 64), (3, 1500, 64)])
def test_states_keep_every_part(dtype, in_place, heads, L, d):
    """One token of each head, in all places of a chunk and in all segments."""
    P = need_gpu()
    rng = np.random.default_rng(L)
    at = [(7 * h * L // max(heads, 8) + 11 * h) % L for h in range(heads)]
    slopes = np.full(heads, min(1e-3, 0.9 / L), np.float32)
    k, v, q = np.zeros((heads, L, d), np.float32), np.zeros((heads, d, (L + 7) // 8 * 8), np.float32), _bf16(rng, heads, L, d)
    one = [_bf16(rng, heads, d) if dtype == "bf16" else rng.standard_normal((heads, d)).astype(np.float32) for _ in range(2)]
    for h in range(heads):
        k[h, at[h]] = one[0][h]
    v[:, :, :L] = _bf16(rng, heads, d, L)
    for h in range(heads):
        v[h, :, at[h]] = one[1][h]
    qd, kd, vd = (torch.from_numpy(t).cuda().to(DT[dtype]) for t in (q, k, v))
    o = torch.empty((L, heads * d), dtype=DT[dtype], device="cuda")
    zero = torch.zeros((heads, d, d), device="cuda")
    out = zero if in_place else torch.empty_like(zero)
    P.linear_attention(qd, kd, vd, torch.from_numpy(slopes).cuda(), o, state_in=zero, state_out=out)
    ref = _state(*one, slopes, at, L)
    bound = (math.ceil(L / 64) + 24) * U * np.abs(ref)
    assert_elementwise(out.double().cpu().numpy(), ref, bound + 1e-40, 0.0, f"{dtype} {heads}x{L}x{d}")
