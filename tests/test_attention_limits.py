"""osd_tree_attention refuses what its counters and exponents cannot hold (no GPU needed)."""
import pytest

from tests.test_cache_abi import P, attention


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_a_scale_that_leaves_fp32_with_the_exponent_base(scale):
    """scale log2(e) is what scores are multiplied by."""
    assert attention(scale=scale) == -1
