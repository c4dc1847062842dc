"""Pins of the 8-bit block's oracle: e4m3 against torch's type, scales and
products by hand, rotations against complex numbers and their own invariants."""
import numpy as np
import pytest
import torch

from oracle import fp8_block as B


def test_values_are_torchs():
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(B.VALUES, t, equal_nan=True)


def test_rounding_is_torchs():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.6, 20000), B.VALUES[:127],
                        (B.VALUES[:126] + B.VALUES[1:127]) / 2, -(B.VALUES[:126] + B.VALUES[1:127]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(B.to_e4m3(x), t)
    assert B.to_e4m3(1e9) == 448 and B.to_e4m3(-500.0) == -448


def test_scales_by_hand():
    x = np.zeros((3, 160), np.float32)
    x[0, 5], x[0, 130] = 448.0, -896.0
    x[1, :128] = 7.0
    codes, scales = B.quantize_rows(x)
    assert scales[:, 0].tolist() == [1.0, 2.0] and codes[0, 5] == 448 and codes[0, 130] == -448
    assert scales[0, 1] == np.float32(7.0) / np.float32(448.0) and (codes[1, :128] == 448).all()
    assert (scales[:, 2] == np.float32(2.0 ** -126)).all() and not codes[2].any()
    w = np.zeros((144, 130), np.float32)
    w[143, 129], w[0, 0] = -4.48, 44.8
    codes, scales = B.quantize_weight(w)
    assert codes.shape == (130, 144) and codes[129, 143] == -448 and codes[0, 0] == 448
    assert scales[1, 1] == np.float32(4.48) / np.float32(448) and scales[0, 1] == np.float32(2.0 ** -126)


def test_values_and_product():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 300)), rng.standard_normal((300, 7))
    a, b = B.rows_values(*B.quantize_rows(x)), B.weight_values(*B.quantize_weight(w))
    assert np.all(np.abs(a - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * 4 / 448)
    y = B.linear(a, b, bias=np.arange(7.0))
    want = [[sum(a[i, k] * b[j, k] for k in range(300)) + j for j in range(7)] for i in range(5)]
    assert np.allclose(y, want, rtol=1e-12)
    assert np.allclose(B.linear(a, b, gate=np.full(7, 2.0), residual=np.ones((5, 7))), 1 + 2 * (y - np.arange(7.0)))
    t = torch.from_numpy(y)
    assert np.allclose(B.linear(a, b, bias=np.arange(7.0), gelu=True),
                       torch.nn.functional.gelu(t, approximate="tanh").numpy(), atol=1e-14)


def test_ln_modulate_is_torchs():
    rng = np.random.default_rng(2)
    x, sh, sc = rng.standard_normal((6, 48)), rng.standard_normal((3, 48)), rng.standard_normal((3, 48))
    n = torch.nn.functional.layer_norm(torch.from_numpy(x), (48,), eps=1e-6).numpy()
    assert np.allclose(B.ln_modulate(x, sh, sc, 2), n * (1 + np.repeat(sc, 2, 0)) + np.repeat(sh, 2, 0))


@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
def test_rotation(pairs):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 2 * 16))
    pos, sections = rng.integers(0, 50, (3, 4)), (2, 3, 1)
    freqs = rng.uniform(0.01, 1, 6)
    y = B.heads(x, 2, pos, freqs, sections, pairs)
    axis = [0, 0, 1, 1, 1, 2]
    turn = np.exp(1j * pos[axis].T * freqs)                                  # [tokens, pairs]
    z = x.reshape(4, 2, 16)
    first, second = (slice(0, 12, 2), slice(1, 12, 2)) if pairs == "adjacent" else (slice(0, 6), slice(6, 12))
    w = (z[..., first] + 1j * z[..., second]) * turn[:, None]
    assert np.allclose(y[..., first], w.real.transpose(1, 0, 2)) and np.allclose(y[..., second], w.imag.transpose(1, 0, 2))
    assert np.array_equal(y[..., 12:], z[..., 12:].transpose(1, 0, 2))
    # q . k goes by the difference of the positions alone, and the origin turns by nothing
    q, k = (rng.standard_normal((1, 16)) for _ in range(2))

    def dot(a, b):
        r = [B.heads(v, 1, np.full((3, 1), p), freqs, sections, pairs)[0, 0] for v, p in ((q, a), (k, b))]
        return r[0] @ r[1]
    assert np.isclose(dot(7, 3), dot(104, 100)) and not np.isclose(dot(7, 3), dot(7, 4))
    assert np.array_equal(B.heads(q, 1, np.zeros((3, 1)), freqs, sections, pairs)[0], q)


def test_norms():
    rng = np.random.default_rng(4)
    x, w, b = rng.standard_normal((5, 3 * 8)), rng.standard_normal(8), rng.standard_normal(8)
    none = (np.zeros((1, 5)), np.ones(1), (1,))
    t = torch.from_numpy(x).reshape(5, 3, 8)
    ln = torch.nn.functional.layer_norm(t, (8,), torch.from_numpy(w), torch.from_numpy(b), 1e-6)
    assert np.allclose(B.heads(x, 3, *none, norm="layer", weight=w, bias=b), ln.permute(1, 0, 2).numpy())
    rms = t / (t.square().mean(2, keepdim=True) + 1e-6).sqrt() * torch.from_numpy(w)
    assert np.allclose(B.heads(x, 3, *none, norm="rms", weight=w, scale=2.0), 2 * rms.permute(1, 0, 2).numpy())
    row, wide = torch.from_numpy(x), rng.standard_normal(24)
    row = row / (row.square().mean(1, keepdim=True) + 1e-6).sqrt() * torch.from_numpy(wide)
    assert np.allclose(B.heads(x, 3, *none, norm="rms_row", weight=wide), row.reshape(5, 3, 8).permute(1, 0, 2).numpy())
