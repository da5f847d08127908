"""osd_cache_keep refuses layers that share memory, where one thread would write a row
that another has still to read (no GPU needed), and takes layers that lie in any other way."""
import numpy as np
import pytest

from tests.test_cache_abi import P, keep

PAGE = 2 * 16 * 64  # elements of a page of the call that keep() makes; it has 8 pages and 2 layers


@pytest.mark.parametrize("kw", [
    dict(ls=0), dict(ls=PAGE - 8), dict(ls=8),                      # less than a page apart
    dict(ls=PAGE), dict(ls=7 * PAGE), dict(ls=7 * PAGE + 8),        # pages one after another: a page of the next layer's
    dict(ls=8 * PAGE - 8),                                          # the last page's end
    dict(ps=4 * PAGE, ls=PAGE, layers=5), dict(ps=4 * PAGE, ls=3 * PAGE + 8),  # layers inside a page's distance: too many, too far
    dict(ps=3 * PAGE, ls=4 * PAGE, layers=4),                       # only the first and the last layer meet
    dict(ps=1 << 40, ls=0, layers=65535, pages=1 << 30),
])
def test_layers_that_share_memory_are_refused(kw):
    assert keep(vc=P(0x10000000), **kw) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["layers apart", "layers in a page", "one page, any distance"])
def test_layers_apart_are_taken(layout):
    import torch
    import paper_2310_07177_amd as osd
    from oracle import cache_ref as ref
    from tests._cache_helpers import f64
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


def test_an_expanded_tensor_is_refused():
    """The check is the C ABI's: what the binding passes for one memory of three layers."""
    assert keep(vc=P(0x10000000), ls=0, layers=3) == -1
