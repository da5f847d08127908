"""osd_tree_attention of heads that do not fill their tiles: what lies behind a head in LDS
changes neither what comes out nor what the call does for it."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import Cache, check_attention, dev, f64, torch_dtype, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,G", [(2, 4), (10, 4), (31, 4), (64, 4)])
def test_every_head_size(osd, N, G, dtype):
    for D in range(8, 257, 8):
        g = np.random.default_rng(D)
        lens = [90, 3]
        c = Cache(g, lens, N, 1, D, 16, dtype)
        q, parent = dev(g.normal(0, 1, (2, N, G, D)).astype(np.float32), torch_dtype(dtype)), trees(g, 2, N)
        got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent))
        want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, D ** -0.5, parent)
        check_attention(got, want, mass, reach, 90 + N, dtype, str(D))


def least(osd, D, dtype):
    """The shortest of some replays of ten calls of 64 nodes over 2000 tokens."""
    import torch
    g = np.random.default_rng(1)
    c = Cache(g, [2000] * 16, 64, 8, D, 16, dtype)
    q, parent = dev(g.normal(0, 1, (16, 64, 16, D)).astype(np.float32), torch_dtype(dtype)), dev(trees(g, 16, 64))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    times = []
    with torch.cuda.stream(side):
        osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
        with torch.cuda.graph(graph, stream=side):
            for _ in range(10):
                osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
        for _ in range(8):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record(side)
            graph.replay()
            b.record(side)
            side.synchronize()
            times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,like", [(72, 80), (40, 64), (136, 256)])
def test_a_smaller_head_does_not_take_twice_as_long(osd, D, like, dtype):
    """It has less to read and to compute than the one that fills the same tiles.  (With what lies
    behind it counted, it took two to four times as long.)"""
    assert least(osd, D, dtype) < 2 * least(osd, like, dtype)
