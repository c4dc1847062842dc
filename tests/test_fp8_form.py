"""The rule that chooses the tile and the parts of K of a product of e4m3 operands (host code): what
it takes at sizes measured on an MI355X, and the bounds the launches rely on."""
import random

import pytest

from fp8_form_util import TILES, fp8_form
from paper_2607_12358_amd import _lib as L


# rows, outputs, inputs and measured microseconds: tiles of 256, 128 and 64, and the best in parts
@pytest.mark.parametrize("m,n,k,us,parts", [
    (64, 1536, 8960, (88.5, 40.8, 27.5), 11.9), (300, 1536, 8960, (91.6, 42.0, 27.9), 18.3), (17, 8960, 1536, (20.2, 10.6, 7.9), None),
    (600, 4608, 1536, (22.9, 11.6, 11.2), None), (2500, 4608, 8960, (104.4, 108.5, 173.0), None), (4096, 4608, 1536, (47.5, 35.9, 52.3), None),
    (8200, 1536, 8960, (110.2, 128.8, 190.3), None)])
def test_fastest_measured_form_is_taken(m, n, k, us, parts):
    tile, split, _ = fp8_form(m, n, k)
    if parts is None:
        assert split == 1 and us[TILES.index(tile) - 1] <= 1.05 * min(us), (tile, us)
    else:
        assert split > 1 and parts < min(us)


def test_bounds():
    """Few rows have their own kernel; a split's items stay within two rounds, each with two blocks of
    128 inputs at least; exact products take no 256 x 256 tiles; the library reports what they need."""
    rng = random.Random(3)
    occ, side = {"256x256": 1, "128x128": 2, "64x64": 4}, {"256x256": 256, "128x128": 128, "64x64": 64}
    seen = set()
    lib = L.lib()
    for _ in range(20000):
        m, n, k = int(2 ** rng.uniform(0, 18)), int(2 ** rng.uniform(0, 15)), 16 * int(2 ** rng.uniform(0, 11))
        cus = rng.choice((256, 256, 304, 64))
        most = 0
        for exact in (False, True):
            tile, split, floats = fp8_form(m, n, k, exact, cus)
            seen.add((tile, exact, split > 1))
            assert (tile == "rows") == (m <= 16 or m <= 32 and -(-n // 16) < 2 * cus) and (split == 1 or tile not in ("rows", "256x256"))
            assert not (exact and tile == "256x256")
            most = max(most, floats)
            if split == 1:
                assert floats == 0
                continue
            s = side[tile]
            tiles = -(-m // s) * -(-n // s)
            assert floats == tiles * split * s * s and tiles * split <= 2 * cus * occ[tile] and -(-k // 128) >= 2 * split
        if cus == 256:
            assert lib.acid_linear_fp8_workspace_needed(m, n, k) == 4 * most
    assert len(seen) == 2 + 1 + 4 + 4  # rows; 256; 128 and 64, exact or not, split or not


def test_exact_products_of_many_rows():
    assert fp8_form(32760, 4608, 1536)[0] == "256x256" and fp8_form(32760, 4608, 1536, True)[0] == "128x128"
