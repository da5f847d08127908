"""osd_tree_attention of bf16 values is as exact as fp32 probabilities allow, but for the
output's own rounding.

A probability enters the second product as two bf16 numbers: its upper half (cut, so less
than 2^-7 of it is left) and what is left, rounded (by at most 2^-8 of that, 2^-15 of the
probability; 2^-23 of it is added on the way).  That is 2^-15 + 2^-22 relative to sum p |v|,
beside what fp32 scores and exponentials give (as in _cache_helpers) and the sums, of twice
as many terms."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import E, HALF, Cache, dev, f64, torch_dtype, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("lens,N,Hq,H,D", [([0, 1, 300], 1, 8, 2, 128), ([2500], 1, 8, 1, 64), ([700, 90], 4, 4, 1, 256),
                                           ([50, 413], 3, 10, 2, 80), ([1000, 129], 12, 8, 2, 128), ([3000], 64, 2, 1, 128),
                                           ([500, 333], 32, 4, 1, 64), ([700, 20], 64, 4, 1, 128), ([900], 60, 4, 1, 64),
                                           ([640, 7], 33, 4, 1, 256), ([411, 96], 40, 4, 1, 96), ([150] * 70, 20, 8, 2, 128)])
def test_probabilities_keep_their_bits(osd, lens, N, Hq, H, D):
    g = np.random.default_rng(N + D)
    B = len(lens)
    c = Cache(g, lens, N, H, D, 16, "bf16")
    q, parent = dev(g.normal(0, 1, (B, N, Hq, D)).astype(np.float32), torch_dtype("bf16")), trees(g, B, N)
    got = f64(osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent)))
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, D ** -0.5, parent)
    n = max(lens) + N
    r = (D + 5) * E * reach[..., None] + 2 * E + (n + 3 * n / 32 + 8) * E
    tol = (2 * r + n * E + 2.0 ** -15 + 2.0 ** -22) * mass * 1.01 + HALF["bf16"] * np.abs(want)
    over = np.abs(got - want) / tol
    print("largest error, of its bound:", over.max(), flush=True)
    assert (over <= 1).all(), np.unravel_index(over.argmax(), over.shape)
