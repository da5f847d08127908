"""osd_cache_keep takes layers that lie in any way in which they share no memory."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["layers apart", "layers in a page", "one page, any distance"])
def test_layers_apart_are_taken(layout):
    import torch
    import paper_2310_07177_amd as osd
    g = np.random.default_rng(3)
    L, P_, H, S, D, N = 3, 1 if layout.startswith("one") else 4, 2, 8, 16, 6
    if layout == "layers apart":
        k, v = (torch.randn(L, 2, P_, H, S, D, device="cuda").bfloat16().unbind(1)[0] for _ in range(2))
    elif layout == "layers in a page":
        k, v = torch.randn(P_, L, 2, H, S, D, device="cuda").bfloat16().transpose(0, 1).unbind(2)
    else:
        k, v = torch.randn(L, 2, 1, H, S, D, device="cuda").bfloat16().unbind(1)
    table = g.permutation(P_)[None].astype(np.int32)
    lens = np.array([1 if P_ == 1 else 13], np.int32)
    path, acc = np.array([[2, 3, 5, -1, -1, -1]], np.int32), np.array([3], np.int32)
    wk, wv = f64(k).copy(), f64(v).copy()
    dev = lambda a: torch.from_numpy(a).cuda()
    new = osd.osd_cache_keep(k, v, dev(table), dev(lens), dev(path), dev(acc))
    assert new.tolist() == ref.keep(wk, wv, table, lens, path, acc).tolist()
    assert np.array_equal(f64(k), wk) and np.array_equal(f64(v), wv)
