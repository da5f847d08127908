"""osd_tree_attention of one long context among short ones: its units are shared by most
of the workgroups, more than 64 of them, in a row or cut apart."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import Cache, check_attention, dev, f64, torch_dtype, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,long,N,Hq,H,D", [(70, 60000, 1, 4, 1, 64), (70, 12000, 16, 2, 1, 128), (66, 12000, 40, 2, 1, 64),
                                             (8, 60000, 2, 4, 1, 64), (8, 12000, 30, 2, 1, 128), (300, 3000, 5, 4, 1, 256),
                                             (40, 6000, 9, 14, 7, 64)])
def test_one_long_context(B, long, N, Hq, H, D, dtype):
    import torch
    import paper_2310_07177_amd as osd
    g = np.random.default_rng(B + N)
    lens = [int(x) for x in g.integers(0, 60, B)]
    lens[B // 3] = long
    c = Cache(g, lens, N, H, D, 16, dtype)
    q, parent = dev(g.normal(0, 1, (B, N, Hq, D)).astype(np.float32), torch_dtype(dtype)), trees(g, B, N)
    got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent))
    again = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent))
    assert torch.equal(got, again)
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, D ** -0.5, parent)
    check_attention(got, want, mass, reach, long + N, dtype)
