"""The parts of K that the rule for e4m3 products takes, against the measured times of all its choices."""
import pytest

from fp8_form_util import fp8_form

# Microseconds on one MI355X of 256 CUs, in a graph, weights in turn: tile and parts
BF16 = {
    (64, 1536, 8960): ({"256x256": {1: 89.5}, "128x128": {1: 42.0}, "64x64": {1: 28.6, 2: 18.6, 4: 13.2, 6: 12.1, 8: 11.5, 12: 12.7}}, "64x64", 12),
    (300, 1536, 8960): ({"256x256": {1: 92.7}, "128x128": {1: 42.8}, "64x64": {1: 29.1, 2: 20.8, 4: 17.8, 6: 18.8, 8: 19.6, 12: 20.8}}, "64x64", 4),
    (600, 4608, 1536): ({"256x256": {1: 23.4}, "128x128": {1: 11.8, 2: 26.9}, "64x64": {1: 11.5, 2: 25.3}}, "64x64", 1),
    (2048, 1536, 8960): ({"256x256": {1: 93.5}, "128x128": {1: 44.1, 2: 48.0, 3: 53.3}, "64x64": {1: 47.0, 2: 57.9}}, "128x128", 2),
    (2500, 4608, 8960): ({"256x256": {1: 102.3}, "128x128": {1: 114.2, 2: 155.9}, "64x64": {1: 182.5}}, "256x256", 1),
    (4096, 4608, 1536): ({"256x256": {1: 47.2}, "128x128": {1: 36.8, 2: 101.5}, "64x64": {1: 53.6}}, "128x128", 1),
    (8200, 1536, 8960): ({"256x256": {1: 109.0}, "128x128": {1: 131.2, 2: 159.5}, "64x64": {1: 191.1}}, "256x256", 1)}
EXACT = {
    (64, 1536, 8960): ({"128x128": {1: 74.3}, "64x64": {1: 46.5, 4: 18.2, 8: 14.0, 12: 14.9}}, "64x64", 12),
    (300, 1536, 8960): ({"128x128": {1: 75.7}, "64x64": {1: 47.6, 4: 24.6, 8: 24.1, 12: 24.5}}, "64x64", 4)}


@pytest.mark.parametrize("size", BF16)
def test_parts(size):
    times, tile, split = BF16[size]
    assert fp8_form(*size)[:2] == (tile, split)
    assert times[tile][split] <= 1.11 * min(min(t.values()) for t in times.values())


@pytest.mark.parametrize("size", EXACT)
def test_parts_of_exact_products(size):
    times, tile, split = EXACT[size]
    assert fp8_form(*size, True)[:2] == (tile, split)
    assert times[tile][split] <= 1.28 * min(min(t.values()) for t in times.values())
