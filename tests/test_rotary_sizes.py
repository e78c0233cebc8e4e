"""How many threads a rotation takes, on the host, where its heads pass 32 bits: what the entry points refuse a call by."""
import pytest

from paper_2411_17686_amd import ficoco as fc
from tests.plan_hook import rotate_threads

LIMIT = 2 ** 31 - 1


@pytest.mark.parametrize("heads", [LIMIT, LIMIT - 1, LIMIT - 2, LIMIT - 3, LIMIT // 2 + 1])
@pytest.mark.parametrize("B,n", [(1, 1), (1, 7), (1000, 1), (32767, 1 << 30)])
@pytest.mark.parametrize("d,norm", [(64, fc.NORM_NONE), (128, fc.NORM_RMS)])
def test_heads_that_pass_32_bits_count(B, n, heads, d, norm):
    """A row has a lane at least, and lanes go through four heads at most."""
    for dtype in (fc.F32, fc.BF16):
        assert rotate_threads(B, n, heads, 0, d, d, norm, dtype, dtype) >= min(B * n * -(-heads // 4) * 4, LIMIT)


def test_ordinary_calls():
    """Rows of chunks of 8 (bfloat16) or 4, one slot of two chunks a lane; items of one head, or of four from 3 M features on."""
    assert rotate_threads(1, 1, 32, 8, 128, 128, fc.NORM_NONE, fc.BF16, fc.BF16) == 40 * 8
    assert rotate_threads(2, 3, 5, 0, 64, 64, fc.NORM_NONE, fc.F32, fc.F32) == 2 * 3 * 5 * 8
    assert rotate_threads(8, 1000, 30, 2, 128, 128, fc.NORM_NONE, fc.BF16, fc.BF16) == 8000 * (8 + 1) * 8
