"""osd_tree_attention against the 64-bit reference: sizes, head layouts, pages,
trees, padding, what lies in masked places, workspaces, streams and graphs."""
import math

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


def queries(g, B, N, Hq, D, dtype, std=1.0):
    return dev(g.normal(0, std, (B, N, Hq, D)).astype(np.float32), torch_dtype(dtype))


def parity(osd, g, lens, N, Hq, H, D, S, dtype, tree, new=None, scale=None, std=1.0, label="", **kw):
    import torch
    B = len(lens)
    c = Cache(g, lens, N, H, D, S, dtype, **kw)
    q = queries(g, B, N, Hq, D, dtype, std)
    parent = trees(g, B, N) if tree else None
    out = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, None if parent is None else dev(parent),
                                 None if new is None else dev(np.array(new, np.int32)), scale)
    torch.cuda.synchronize()
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, D ** -0.5 if scale is None else scale,
                                      parent, new)
    check_attention(out, want, mass, reach, max(lens) + N, dtype, label)


SHAPES = [  # lens, N, Hq, H, D, S
    ([0], 1, 1, 1, 64, 16), ([1], 1, 8, 1, 128, 16), ([17, 0, 300], 1, 8, 2, 128, 16), ([5, 700], 9, 4, 4, 64, 32),
    ([31, 32, 33], 16, 4, 1, 128, 16), ([127, 128, 129, 95], 17, 6, 2, 64, 64), ([1000, 13], 64, 4, 2, 128, 16),
    ([257], 64, 8, 1, 64, 24), ([90, 411], 33, 7, 1, 80, 5), ([1500], 5, 16, 1, 256, 16), ([63, 1], 20, 10, 2, 256, 128),
    ([200], 2, 3, 3, 8, 1), ([333, 40], 7, 4, 2, 72, 48), ([2500], 64, 2, 2, 128, 4096), ([600, 601], 3, 64, 4, 136, 16),
    ([120, 4], 64, 20, 2, 40, 7), ([3000, 1, 700], 1, 28, 4, 128, 256), ([100], 64, 40, 1, 128, 16),
]


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[1:])))
def test_parity(osd, shape, dtype, tree):
    lens, N, Hq, H, D, S = shape
    print(shape, dtype, tree, flush=True)
    parity(osd, np.random.default_rng(N * 1000 + D), lens, N, Hq, H, D, S, dtype, tree)


@pytest.mark.parametrize("N", list(range(1, 65, 7)) + [2, 4, 16, 32, 48])
def test_every_number_of_nodes(osd, N):
    parity(osd, np.random.default_rng(N), [N, 129, 64 - N % 3], N, 8, 2, 64, 16, "bf16", True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_around_every_tile(osd, dtype):
    g = np.random.default_rng(7)
    lens = [0, 1, 2, 7, 14, 15, 16, 30, 31, 47, 62, 63, 64, 65, 111, 126, 127, 128, 159, 190, 191, 192, 254, 255, 256, 383, 511]
    parity(osd, g, lens, 2, 4, 1, 64, 16, dtype, False)
    parity(osd, g, lens, 3, 2, 2, 128, 8, dtype, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,std", [(3.0, 6.0), (0.0, 1.0), (-1.0, 1.0), (1e-30, 1.0), (300.0, 1.0)])
def test_scales(osd, dtype, scale, std):
    parity(osd, np.random.default_rng(3), [500, 64], 9, 4, 1, 64, 16, dtype, True, scale=scale, std=std)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hq,H,D", [(1, 4, 1, 64), (16, 4, 2, 128), (64, 4, 1, 128), (30, 8, 2, 256)])
@pytest.mark.parametrize("order", ["rising", "falling", "one far key", "far tree"])
def test_scores_far_apart(osd, order, N, Hq, H, D, dtype):
    """Scores that leave the range of a reference taken from the first keys, in
    either direction, at any place: several hundred powers of two apart."""
    import torch
    g = np.random.default_rng(61)
    lens = [700, 3, 64]
    c = Cache(g, lens, N, H, D, 16, dtype)
    q = queries(g, 3, N, Hq, D, dtype)
    q[..., 0] = 4.0
    parent = trees(g, 3, N)
    for b, n in enumerate(lens):
        for j in range(n + N):
            p, s = c.row(b, j)
            if order == "rising":
                x = j * 0.5
            elif order == "falling":
                x = -j * 0.5
            elif order == "one far key":
                x = 200.0 if j == max(n - 2, 0) else 0.0
            else:
                x = 150.0 if j == n else -100.0 if j == n + 1 else 0.0
            c.k[p, :, s, 0] = x
    got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent), scale=0.5)
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, 0.5, parent)
    check_attention(got, want, mass, reach, 700 + N, dtype, order)


@pytest.mark.parametrize("lens,N,Hq,H,D", [([9000], 64, 4, 1, 128), ([3000, 40], 64, 16, 2, 64), ([5000], 64, 12, 1, 256),
                                           ([2000] * 3, 33, 32, 1, 128), ([700] * 70, 3, 8, 4, 64), ([300] * 40, 20, 32, 8, 128)])
def test_divisions(osd, lens, N, Hq, H, D):
    """Units cut apart into many parts that are joined together, units in a row, row
    blocks, more sequences than a wave has lanes."""
    g = np.random.default_rng(67)
    new = [int(x) for x in g.integers(1, N + 1, len(lens))]
    parity(osd, g, lens, N, Hq, H, D, 16, "bf16", True, new=new, label=str((len(lens), N, Hq, H, D)))
    if D < 256:
        parity(osd, g, lens[:3], N, Hq, H, D, 8, "f32", True)


def test_many_sequences(osd):
    g = np.random.default_rng(5)
    lens = [int(x) for x in g.integers(0, 200, 300)]
    new = [int(x) for x in g.integers(0, 5, 300)]
    parity(osd, g, lens, 4, 4, 2, 64, 16, "bf16", True, new=new)
    lens = [-1 if x < 0.3 else int(100 * x) for x in g.random(1100)]
    parity(osd, g, lens, 1, 2, 1, 8, 16, "f32", False)


@pytest.mark.parametrize("N,Hq,D,dtype", [(1, 1, 128, "bf16"), (9, 16, 128, "bf16"), (9, 8, 256, "bf16"), (5, 4, 256, "f32")])
def test_the_largest_batch(osd, N, Hq, D, dtype):
    """4096 sequences, most of them padding: the kernels with the most LDS beside the batch's table."""
    g = np.random.default_rng(N + D)
    lens = [int(x) if x >= 0 and g.random() < 0.1 else -1 for x in g.integers(0, 40, 4096)]
    parity(osd, g, lens, N, Hq, 1, D, 16, dtype, N > 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padding_and_invalid_sequences(osd, dtype):
    import torch
    g = np.random.default_rng(11)
    lens = [40, -1, 300, 64, 129, 200, 5, 9, 77]
    new = [6, 6, 0, 1, 3, 7, -2, 5, 6]
    B, N, Hq, H, D = 9, 6, 4, 2, 64
    c = Cache(g, lens, N, H, D, 16, dtype)
    table = c.table.copy()
    table[4, 3] = 10 ** 6      # no such page
    table[8, 4] = -5
    parent = trees(g, B, N)
    parent[0, 2] = 1
    parent[7, 3] = 3           # its own parent
    q = queries(g, B, N, Hq, D, dtype)
    out = torch.full((B, N, Hq, D), 7.0, device="cuda", dtype=q.dtype)
    got = osd.osd_tree_attention(q, c.k, c.v, dev(table), c.d_lens, dev(parent), dev(np.array(new, np.int32)), out=out)
    assert got is out
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), table, lens, D ** -0.5, parent, new)
    assert np.isnan(want[4, :3]).all() and np.isnan(want[5]).all() and np.isnan(want[6]).all()
    assert np.isnan(want[7, :5]).all() and np.isnan(want[8]).all() and (want[1] == 0).all() and (want[2] == 0).all()
    check_attention(got, want, mass, reach, 310, dtype)
    # a context longer than its table
    out = osd.osd_tree_attention(q[:1], c.k, c.v, dev(table[:1, :2]), dev(np.array([30], np.int32)), dev(parent[:1]))
    assert torch.isnan(out).all()
    out = osd.osd_tree_attention(q[:1], c.k, c.v, dev(table[:1, :2]), dev(np.array([2 ** 31 - 1], np.int32)))
    assert torch.isnan(out).all()


@pytest.mark.parametrize("H,Hq", [(1, 1), (1, 4), (2, 16)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_a_node_does_not_see_does_not_reach_it(osd, dtype, what, H, Hq):
    import torch
    g = np.random.default_rng(13)
    N, D, S, lens = 12, 64, 16, [70, 0, 127]
    c = Cache(g, lens, N + 4, H, D, S, dtype, spare=3)
    q = queries(g, 3, N, Hq, D, dtype)
    parent = trees(g, 3, N)
    parent[:, 5:] = np.minimum(parent[:, 5:], 4)          # node 5 is a leaf
    clean = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent))
    used = set(c.table[c.table >= 0].tolist())
    for page in set(range(c.k.shape[0])) - used:
        c.k[page], c.v[page] = what, what
    for b, n in enumerate(lens):
        for j in range(n + N, n + N + 4):                 # behind the last token
            p, s = c.row(b, j)
            c.k[p, :, s], c.v[p, :, s] = what, what
        p, s = c.row(b, n + 5)                            # the leaf: other nodes do not see it
        c.v[p, :, s] = what
        c.k[p, :, s] = what
    got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent))
    others = [n for n in range(N) if n != 5]
    assert torch.equal(got[:, others], clean[:, others])
    assert not torch.isfinite(got[:, 5]).any()
    # a node that others see: exactly they get it
    p, s = c.row(0, lens[0] + 5)
    c.k[p, :, s] = 0.25
    c.v[p, :, s] = 0.5
    p, s = c.row(0, lens[0] + 2)
    c.v[p, 0, s, 7] = what
    got = f64(osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent)))
    for n, line in enumerate(ref.lines(parent[0], N)):
        for h in range(Hq):
            bad = ~np.isfinite(got[0, n, h])
            seen = 2 in line and h < Hq // H
            assert bad[7] == seen and not np.delete(bad, 7).any()
            if seen and what == what:
                assert got[0, n, h, 7] == what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,N,Hq,H,D,S", [([40000], 1, 8, 1, 128, 16), ([9000, 33, 20000], 9, 4, 2, 64, 64),
                                             ([12345], 64, 4, 1, 128, 16), ([7001, 6000], 50, 8, 1, 256, 24),
                                             ([131071], 2, 1, 1, 64, 256)])
def test_every_key_counts_once(osd, dtype, lens, N, Hq, H, D, S):
    """Equal scores: a row's output counts the keys of each residue, exactly
    until the division."""
    import torch
    g = np.random.default_rng(17)
    B = len(lens)
    c = Cache(g, lens, N, H, D, S, dtype)
    parent = trees(g, B, N)
    ones = torch.eye(D, device="cuda", dtype=c.v.dtype)
    for b, n in enumerate(lens):
        j = torch.arange(n + N, device="cuda")
        page = c.d_table[b].long()[j // S]
        c.v[page, :, j % S] = ones[j % D].unsqueeze(1).expand(-1, H, -1)
    q = torch.zeros(B, N, Hq, D, device="cuda", dtype=c.k.dtype)
    got = f64(osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, dev(parent)))
    for b, n in enumerate(lens):
        context = np.bincount(np.arange(n) % D, minlength=D)
        for i, line in enumerate(ref.lines(parent[b], N)):
            count = context + np.bincount([(n + a) % D for a in line], minlength=D)
            want = count / (n + len(line))
            step = 2.0 ** -8 if dtype == "bf16" else 0.0
            # a reciprocal or division (2 units), a product, the output's rounding
            assert (np.abs(got[b, i] - want) <= want * (step + 4 * 2.0 ** -24)).all(), (b, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(osd, dtype):
    """Queries out of one projection, keys and values of a page side by side,
    pages further apart: as contiguous ones, bit for bit."""
    import torch
    g = np.random.default_rng(19)
    B, N, Hq, H, D, S = 3, 5, 8, 2, 80, 16
    c = Cache(g, [50, 129, 7], N, H, D, S, dtype, shared=True)
    x = queries(g, B, N, Hq + 2 * H, D, dtype)
    parent = dev(trees(g, B, N))
    q = x[:, :, :Hq]
    assert not q.is_contiguous() and not c.k.is_contiguous()
    a = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
    b = osd.osd_tree_attention(q.contiguous(), c.k.contiguous(), c.v.contiguous(), c.d_table, c.d_lens, parent)
    assert torch.equal(a, b)
    one = osd.osd_tree_attention(x[:, :1, :Hq], c.k, c.v, c.d_table, c.d_lens)
    two = osd.osd_tree_attention(x[:, :1, :Hq].contiguous(), c.k, c.v, c.d_table, c.d_lens)
    assert torch.equal(one, two)


def test_pages_beyond_four_gigabytes(osd):
    import torch
    g = np.random.default_rng(23)
    S, D, N, n = 256, 128, 3, 700
    pages = 2 ** 31 // (S * D) + 2600    # over 2^31 elements
    k = torch.empty(pages, 1, S, D, device="cuda", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    c = Cache(g, [n], N, 1, D, S, "bf16")
    far = np.array([[pages - 1, 3, pages - 2]], np.int32)
    for i in range(3):
        k[far[0, i]], v[far[0, i]] = c.k[c.table[0, i]], c.v[c.table[0, i]]
    q = queries(g, 1, N, 4, D, "bf16")
    a = osd.osd_tree_attention(q, k, v, dev(far), c.d_lens)
    b = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens)
    assert torch.equal(a, b)


def test_shared_pages(osd):
    """Two sequences with one prefix, and a page named twice."""
    import torch
    g = np.random.default_rng(29)
    c = Cache(g, [100], 4, 2, 64, 16, "bf16")
    q = queries(g, 1, 4, 4, 64, "bf16")
    one = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens)
    both = osd.osd_tree_attention(q.repeat(2, 1, 1, 1), c.k, c.v, c.d_table.repeat(2, 1), c.d_lens.repeat(2))
    assert torch.equal(both[0], both[1])
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, [100], 0.125)
    check_attention(both[:1], want, mass, reach, 104, "bf16")
    check_attention(one, want, mass, reach, 104, "bf16")
    table = np.where(c.table >= 0, c.table[0, 0], -1).astype(np.int32)
    got = osd.osd_tree_attention(q, c.k, c.v, dev(table), c.d_lens)
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), table, [100], 0.125)
    check_attention(got, want, mass, reach, 104, "bf16")


def test_equal_calls_and_workspaces_across_sizes(osd):
    """Calls of other sizes between equal ones leave nothing behind."""
    import torch
    g = np.random.default_rng(31)
    cases = [([3000, 10, 500], 33, 8, 2, 64, 16, "bf16"), ([20000], 1, 8, 1, 128, 16, "bf16"),
             ([50] * 40, 3, 4, 2, 256, 16, "f32"), ([5000], 64, 8, 1, 128, 64, "bf16"), ([1], 1, 1, 1, 8, 16, "f32")]
    calls = []
    for lens, N, Hq, H, D, S, dtype in cases:
        c = Cache(g, lens, N, H, D, S, dtype)
        calls.append((queries(g, len(lens), N, Hq, D, dtype), c.k, c.v, c.d_table, c.d_lens, dev(trees(g, len(lens), N))))
    first = [osd.osd_tree_attention(*a) for a in calls]
    for order in ([4, 3, 2, 1, 0], [1, 1, 3, 0, 2, 4, 3]):
        for i in order:
            assert torch.equal(osd.osd_tree_attention(*calls[i]), first[i]), i


def test_streams(osd):
    """Inputs made on one stream, calls on two others at once."""
    import torch
    g = np.random.default_rng(37)
    c = Cache(g, [4000, 900], 8, 2, 128, 16, "bf16")
    q, parent = queries(g, 2, 8, 8, 128, "bf16"), dev(trees(g, 2, 8))
    want = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(20):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_graph_serves_other_lengths(osd):
    """A captured call, replayed with other lengths, pages and trees, eager
    calls between the replays; two graphs of one stream."""
    import torch
    g = np.random.default_rng(41)
    B, N, Hq, H, D, S = 3, 16, 8, 2, 64, 16
    c = Cache(g, [2000, 2000, 2000], N, H, D, S, "bf16")
    q, parent, lens = queries(g, B, N, Hq, D, "bf16"), dev(trees(g, B, N)), c.d_lens.clone()
    call = lambda: osd.osd_tree_attention(q, c.k, c.v, c.d_table, lens, parent)
    side = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(side):
        call()
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs.append(call())
            graphs.append(graph)
        for i, now in enumerate([[2000, 0, 17], [5, 1999, 600], [-1, 128, 127], [2000, 2000, 2000], [0, 0, 0], [31, 1000, 1500]]):
            lens.copy_(torch.tensor(now, dtype=torch.int32))
            parent.copy_(torch.from_numpy(trees(g, B, N)))
            q.copy_(queries(g, B, N, Hq, D, "bf16"))
            graphs[i % 2].replay()
            graphs[1 - i % 2].replay()
            eager = call()
            side.synchronize()
            assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager), now
            want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, now, D ** -0.5, parent.cpu().numpy())
            check_attention(eager, want, mass, reach, 2016, "bf16", str(now))


def test_capture_without_an_earlier_call(osd):
    import torch
    g = np.random.default_rng(43)
    c = Cache(g, [3000], 2, 1, 64, 16, "f32")
    q = queries(g, 1, 2, 4, 64, "f32")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens)
        for _ in range(3):
            out.zero_()
            graph.replay()
            side.synchronize()
            want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, [3000], 0.125)
            check_attention(out, want, mass, reach, 3002, "f32")


def test_outputs_alone_are_written(osd):
    """Guards around the output, and the inputs, stay as they were."""
    import torch
    g = np.random.default_rng(47)
    B, N, Hq, H, D = 2, 3, 4, 2, 40
    c = Cache(g, [77, 200], N, H, D, 16, "bf16")
    q = queries(g, B, N, Hq, D, "bf16")
    n = B * N * Hq * D
    room = torch.full((n + 128,), 3.0, device="cuda", dtype=torch.bfloat16)
    before = [t.clone() for t in (q, c.k, c.v, c.d_table, c.d_lens)]
    osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, out=room[64:64 + n].view(B, N, Hq, D))
    assert (room[:64] == 3).all() and (room[64 + n:] == 3).all()
    assert all(torch.equal(a, b) for a, b in zip(before, (q, c.k, c.v, c.d_table, c.d_lens)))
