"""osd_tree_attention refuses what its counters and exponents cannot hold (no GPU needed)."""
import pytest

from tests.test_cache_abi import P, attention


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_a_scale_that_leaves_fp32_with_the_exponent_base(scale):
    """scale log2(e) is what scores are multiplied by."""
    assert attention(scale=scale) == -1


@pytest.mark.parametrize("kw", [
    dict(B=4096, T=1 << 20, S=16), dict(B=64, T=1 << 26, S=16), dict(B=33, T=1 << 26, S=16),
])
def test_more_tokens_than_tiles_are_counted(kw):
    """2^35 tokens are 2^30 tiles of 32 keys; twice as many would leave 31 bits."""
    assert attention(ps=1 << 30, out=P(1 << 32), **kw) == -1
