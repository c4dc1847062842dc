"""Pins of the linear-attention block's plain definitions (CPU)."""
import numpy as np
import pytest

from oracle import linear_block as B


def test_attention_equals_its_quadratic_form():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 2, 9, 4))
    S0, slopes = rng.standard_normal((2, 4, 4)), np.array([0.3, 0.0])
    o, S = B.linear_attention(q, k, v, slopes, S0, scale=0.5)
    i = np.arange(9)
    for h in range(2):
        lam = np.exp(-slopes[h])
        p = np.tril(lam ** (i[:, None] - i[None, :])) * (q[h] @ k[h].T)
        ref = 0.5 * (p @ v[h] + lam ** (i + 1)[:, None] * (q[h] @ S0[h]))
        np.testing.assert_allclose(o[:, 4 * h:4 * h + 4], ref, rtol=1e-12)
        np.testing.assert_allclose(S[h], lam ** 9 * S0[h] + (k[h] * lam ** (8 - i)[:, None]).T @ v[h],
                                   rtol=1e-12)


def test_attention_continues_from_its_state():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 2, 7, 4))
    sl = np.array([0.1, 2.0])
    o, S = B.linear_attention(q, k, v, sl)
    o1, S1 = B.linear_attention(q[:, :3], k[:, :3], v[:, :3], sl)
    o2, S2 = B.linear_attention(q[:, 3:], k[:, 3:], v[:, 3:], sl, S1)
    np.testing.assert_array_equal(np.concatenate([o1, o2]), o)
    np.testing.assert_array_equal(S2, S)


def test_seam_is_ln_modulate_after_a_gated_residual():
    import oracle as O
    rng = np.random.default_rng(2)
    h, y = rng.standard_normal((2, 5, 8))
    g, sh, sc = rng.standard_normal((3, 8))
    h1, out = B.residual_norm(h, y, gate=g, shift=sh, scale=sc)
    np.testing.assert_allclose(h1, h + g * y, rtol=1e-12)
    np.testing.assert_allclose(out, O.layer_norm(h1) * (1 + sc) + sh, rtol=1e-9, atol=1e-12)


def test_seam_uses_each_rows_modulation():
    rng = np.random.default_rng(3)
    h, y = rng.standard_normal((2, 5, 8))
    g = rng.standard_normal((3, 8))
    h1, _ = B.residual_norm(h, y, res_scale=0.5, post="rms", gate=g, rows_per_mod=2)
    for r in range(5):
        n = y[r] / np.sqrt(np.mean(y[r] ** 2) + 1e-6)
        np.testing.assert_allclose(h1[r], 0.5 * h[r] + g[r // 2] * n, rtol=1e-12)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_w4_layout_round_trip_and_error(group):
    rng = np.random.default_rng(4)
    w = rng.standard_normal((256, 19)).astype(np.float32)
    w[:group, 3] = 0
    codes, scales = B.w4_quantize(w, group)
    packed, s = B.w4_pack(codes, scales)
    got = B.w4_weights(packed, s, 19)
    want = (codes.astype(float) - 8) * np.repeat(scales.astype(float), group, 1)
    np.testing.assert_array_equal(got, want)
    assert (got[3, :group] == 0).all()
    # rounding to nearest: half a step
    assert (np.abs(got - w.T) <= 0.5001 * np.repeat(scales, group, 1)).all()


def test_w4_layout_places_one_code():
    """Input 41 of output 17 with K = 128: tile 1, run 16 + 1, word 1, second
    octet's element 1 = nibble 4 (low half of byte 2)."""
    codes = np.full((18, 128), 8, np.uint8)
    codes[17, 41] = 5
    packed, _ = B.w4_pack(codes, np.ones((18, 1), np.float32))
    diff = np.argwhere(packed != 0x88)
    assert diff.tolist() == [[1, 0, 17, 6]]
    assert packed[1, 0, 17, 6] == 0x85
