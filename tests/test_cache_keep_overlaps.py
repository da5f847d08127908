"""osd_cache_keep refuses layers that share memory, where one thread would write a row
that another has still to read (no GPU needed)."""
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


def test_an_expanded_tensor_is_refused():
    """The check is the C ABI's: what the binding passes for one memory of three layers."""
    assert keep(vc=P(0x10000000), ls=0, layers=3) == -1


@pytest.mark.parametrize("kw", [
    dict(acc=P(0x90000)), dict(acc=P(0x8fffc)), dict(acc=P(0x90004)),                        # B = 2: 8 bytes each
    dict(path=P(0x90000)), dict(path=P(0x90000 - 20)), dict(path=P(0x90004)),                # 24 bytes
    dict(table=P(0x90000)), dict(table=P(0x90000 - 28)),                                     # 32 bytes
])
def test_new_lengths_over_what_is_read_are_refused(kw):
    """One workgroup of a sequence would write them while others have still to read the path."""
    assert keep(vc=P(0x10000000), **kw) == -1
