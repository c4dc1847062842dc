"""Where the 8-bit block's calls end: the largest launch is below 2^32 threads.  Sizes that pass are seen
by the refusal that comes after, of an address that is not aligned: nothing is launched here."""
import pytest

from paper_2607_12358_amd import _lib as L

G = 1 << 40


# rows and inputs: workgroups of four waves, a wave to 32 rows of one group; 2^24 of them are 2^32 threads
@pytest.mark.parametrize("rows,K,status", [
    (32 * ((1 << 26) - 4), 16, L.ACID_ERR_INVALID_ARG), (32 * ((1 << 26) - 4) + 1, 16, L.ACID_ERR_SHAPE),
    (32 * ((1 << 26) - 1), 128, L.ACID_ERR_SHAPE), (32 * (1 << 26), 128, L.ACID_ERR_SHAPE),
    (32 * ((1 << 25) - 2), 144, L.ACID_ERR_INVALID_ARG), (32 * ((1 << 25) - 1), 144, L.ACID_ERR_SHAPE),
    (32 * ((1 << 11) - 1), 1 << 22, L.ACID_ERR_INVALID_ARG), (32 * (1 << 11), 1 << 22, L.ACID_ERR_SHAPE)])
def test_rows_of_the_largest_launch(rows, K, status):
    lib, ld = L.lib(), (rows + 3) // 4 * 4
    for dtype in (L.ACID_BF16, L.ACID_F32):
        assert lib.acid_quantize_fp8(dtype, rows, K, G + 8, K, 2 * G, K, 3 * G, ld, None) == status
        assert L.last_error()
