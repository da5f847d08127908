"""osd_cache_append and osd_cache_keep against the 64-bit reference, and a whole
step: append, attention, verification, keep."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import E, HALF, Cache, check_attention, dev, f64, torch_dtype, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


def rotation(rows, R, base=10000.0):
    turn = np.arange(rows)[:, None] * base ** (-2.0 * np.arange(R // 2) / R)
    return np.concatenate([np.cos(turn), np.sin(turn)], 1).astype(np.float32)


def rows(g, B, N, H, D, dtype):
    return dev(g.normal(size=(B, N, H, D)).astype(np.float32), torch_dtype(dtype))


def check_rotated(got, want, bound, dtype, label):
    """bound: |x| + |y| of each value's pair."""
    g = f64(got)
    assert np.array_equal(np.isnan(g), np.isnan(want)), label
    tol = 2 * E * bound + HALF[dtype] * np.abs(want)
    assert (np.abs(g - want)[~np.isnan(want)] <= tol[~np.isnan(want)]).all(), label


def pair_sizes(x, R, pairs):
    """|x| + |y| for each value of a head, 0 for what is copied."""
    a = np.zeros_like(x)
    if R:
        i, j = (slice(0, R, 2), slice(1, R, 2)) if pairs else (slice(0, R // 2), slice(R // 2, R))
        a[..., i] = a[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return a


def run_append(osd, g, lens, N, Hq, H, D, S, R, dtype, tree=False, pairs=False, new=None, table=None, fused=False, parent=None,
               in_place=False, turns=None, q_out=None, shared=False, with_q=True):
    import torch
    B = len(lens)
    c = Cache(g, lens, N, H, D, S, dtype, shared=shared)
    table = c.table if table is None else table(c.table.copy())
    if parent is None and tree:
        parent = trees(g, B, N)
    if fused:
        x = rows(g, B, N, Hq + 2 * H, D, dtype)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
    else:
        q, k, v = (rows(g, B, N, h, D, dtype) for h in (Hq, H, H))
    turn = rotation(max(lens) + N if turns is None else turns, R) if R else None
    q0, k0, v0, kc0, vc0 = f64(q), f64(k), f64(v), f64(c.k), f64(c.v)
    got = osd.osd_cache_append(k, v, c.k, c.v, dev(table), c.d_lens, q=q if with_q else None,
                               rotation=None if turn is None else dev(turn), pairs=pairs,
                               parent=None if parent is None else dev(parent),
                               new_len=None if new is None else dev(np.array(new, np.int32)), q_out=q if in_place else q_out)
    torch.cuda.synchronize()
    t64 = None if turn is None else turn.astype(np.float64)
    out, kc, vc = ref.append(q0, k0, v0, kc0, vc0, table, lens, t64, pairs, parent, new)
    if with_q:
        assert (got is q) == in_place
        check_rotated(got, out, pair_sizes(q0, R, pairs), dtype, "q")
        if not R:
            assert np.array_equal(f64(got), out, equal_nan=True)
    else:
        assert got is None
    _, sizes, _ = ref.append(q0, pair_sizes(k0, R, pairs), v0, np.zeros_like(kc0), vc0, table, lens, None, pairs, parent, new)
    if turn is not None:  # (tokens without a position are not written)
        sizes = np.where(kc != kc0, sizes, 0.0)
    check_rotated(c.k, kc, sizes, dtype, "keys")
    same = kc == kc0
    assert np.array_equal(f64(c.k)[same & (sizes == 0)], kc0[same & (sizes == 0)]), "keys that stay"
    assert np.array_equal(f64(c.v), vc), "values"
    if not in_place:
        assert np.array_equal(f64(q), q0) and np.array_equal(f64(k), k0) and np.array_equal(f64(v), v0)


SHAPES = [  # lens, N, Hq, H, D, S, R
    ([0], 1, 1, 1, 64, 16, 64), ([15, 16, 17], 3, 8, 2, 128, 16, 128), ([5, 90], 9, 4, 1, 80, 24, 32), ([7], 2, 2, 2, 80, 5, 20),
    ([100, 3], 20, 6, 2, 64, 32, 6), ([33], 64, 4, 4, 256, 16, 256), ([9, 0], 5, 3, 1, 8, 1, 2), ([2, 60], 4, 4, 2, 72, 16, 24),
    ([1, 2, 3, 4], 33, 40, 8, 128, 64, 64), ([11], 7, 5, 5, 40, 16, 8), ([4], 3, 2, 1, 24, 16, 12), ([700], 2, 64, 64, 256, 16, 254),
]


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[1:])))
def test_append(osd, shape, dtype, pairs):
    lens, N, Hq, H, D, S, R = shape
    print(shape, dtype, pairs, flush=True)
    g = np.random.default_rng(D + N)
    run_append(osd, g, lens, N, Hq, H, D, S, R, dtype, tree=False, pairs=pairs)
    run_append(osd, g, lens, N, Hq, H, D, S, R, dtype, tree=True, pairs=pairs, fused=True, shared=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_variants(osd, dtype):
    g = np.random.default_rng(2)
    run_append(osd, g, [9, 30], 5, 4, 2, 64, 16, 0, dtype)                               # no rotation
    run_append(osd, g, [9, 30], 5, 4, 2, 72, 16, 0, dtype, with_q=False)
    run_append(osd, g, [9, 30], 5, 4, 2, 64, 16, 64, dtype, with_q=False, tree=True)
    run_append(osd, g, [9, 30], 5, 4, 2, 64, 16, 64, dtype, in_place=True)
    run_append(osd, g, [9, 30], 5, 4, 2, 64, 16, 32, dtype, in_place=True, fused=True, tree=True, pairs=True)
    run_append(osd, g, [0, 0, 0], 1000, 4, 2, 64, 64, 64, dtype, new=[1000, 1, 333])      # prompts
    run_append(osd, g, [9, -1, 30, 50, 2, 8], 5, 4, 2, 64, 16, 64, dtype, tree=True, new=[5, 5, 0, 6, -1, 2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_tokens_without_a_place(osd, dtype):
    import torch
    g = np.random.default_rng(3)

    def broken(t):
        t[0, 1] = 999
        t[2, 0] = -1
        return t

    run_append(osd, g, [14, 2, 15, 40], 6, 4, 2, 64, 16, 64, dtype, table=broken)
    run_append(osd, g, [14, 2, 15, 40], 6, 4, 2, 64, 16, 64, dtype, table=lambda t: np.ascontiguousarray(t[:, :1]))
    run_append(osd, g, [14, 2, 15, 40], 6, 4, 2, 64, 16, 64, dtype, turns=17)             # positions that the table lacks
    bad = trees(g, 4, 6)
    bad[1, 3], bad[2, 5], bad[3, 2] = 3, -1, 5
    run_append(osd, g, [14, 2, 15, 40], 6, 4, 2, 64, 16, 64, dtype, parent=bad, new=[6, 6, 5, 4])


def test_append_at_the_largest_length(osd):
    import torch
    g = np.random.default_rng(4)
    c = Cache(g, [14], 6, 2, 64, 16, "f32")
    k = rows(g, 1, 6, 2, 64, "f32")
    before = c.k.clone()
    for n in (2 ** 31 - 1, 2 ** 31 - 3, 32 * c.table.shape[1]):
        q = osd.osd_cache_append(k, k, c.k, c.v, c.d_table, dev(np.array([n], np.int32)), q=k, rotation=dev(rotation(50, 64)))
        assert torch.isnan(q).all() and torch.equal(c.k, before)


def test_append_of_more_tokens_than_a_launch_has_threads_for(osd):
    """2^26 + 5 tokens, a wave each: more than 2^32 threads.  All land where the pages say."""
    import torch
    N, S = (1 << 26) + 5, 1 << 16
    pages = -(-N // S)
    k = torch.randint(-(1 << 15), 1 << 15, (1, N, 1, 8), device="cuda", dtype=torch.int16).view(torch.bfloat16)
    v = torch.randint(-(1 << 15), 1 << 15, (1, N, 1, 8), device="cuda", dtype=torch.int16).view(torch.bfloat16)
    k_cache, v_cache = (torch.zeros(pages, 1, S, 8, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.arange(pages - 1, -1, -1, device="cuda", dtype=torch.int32)[None]
    osd.osd_cache_append(k, v, k_cache, v_cache, table, torch.zeros(1, device="cuda", dtype=torch.int32))
    for cache, x in ((k_cache, k), (v_cache, v)):
        got = cache.flip(0).view(-1, 8).view(torch.int16)
        assert torch.equal(got[:N], x.view(N, 8).view(torch.int16)) and not got[N:].any()


def test_append_graph(osd):
    import torch
    g = np.random.default_rng(5)
    c = Cache(g, [60, 90], 40, 2, 64, 16, "bf16")
    k, v, q = (rows(g, 2, 4, h, 64, "bf16") for h in (2, 2, 4))
    parent, lens, turn = dev(trees(g, 2, 4)), c.d_lens.clone(), dev(rotation(140, 64))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = osd.osd_cache_append(k, v, c.k, c.v, c.d_table, lens, q=q, rotation=turn, parent=parent)
        for i in range(4):
            graph.replay()
            side.synchronize()
            mine, mk, mv = out.clone(), c.k.clone(), c.v.clone()
            eager = osd.osd_cache_append(k, v, c.k, c.v, c.d_table, lens, q=q, rotation=turn, parent=parent)
            assert torch.equal(mine, eager) and torch.equal(mk, c.k) and torch.equal(mv, c.v)
            lens.add_(7)
            parent.copy_(torch.from_numpy(trees(g, 2, 4)))


def paths(g, parent):
    """A path of each tree, and its length."""
    B, N = parent.shape
    out, acc = np.full((B, N), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        line = ref.lines(parent[b], N)[int(g.integers(0, N))][1:]
        out[b, :len(line)], acc[b] = line, len(line)
    return out, acc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,N,H,D,S,layers", [([0], 1, 1, 64, 16, 1), ([7, 0, 31], 64, 2, 128, 16, 3), ([100], 33, 5, 80, 24, 2),
                                                 ([3, 4, 5, 6], 17, 1, 8, 1, 5), ([60, 61], 64, 4, 256, 64, 2)])
def test_keep(osd, dtype, lens, N, H, D, S, layers):
    import torch
    g = np.random.default_rng(N)
    for chain in (False, True):
        c = Cache(g, lens, N, H, D, S, dtype, layers=layers, shared=chain)
        path, acc = paths(g, trees(g, len(lens), N))
        if chain:  # every other node, as long as there are some
            n = (N - 1) // 2
            path[:] = -1
            path[:, :n] = np.arange(2, 2 * n + 1, 2)
            acc[:] = n
        k, v = f64(c.k).copy(), f64(c.v).copy()
        new = osd.osd_cache_keep(c.k, c.v, c.d_table, c.d_lens, dev(path), dev(acc))
        want = ref.keep(k, v, c.table, lens, path, acc)
        assert new.cpu().numpy().tolist() == want.tolist()
        assert np.array_equal(f64(c.k), k) and np.array_equal(f64(c.v), v)
    one = Cache(g, lens, N, H, D, S, dtype)
    k, v = f64(one.k)[None].copy(), f64(one.v)[None].copy()
    osd.osd_cache_keep(one.k, one.v, one.d_table, one.d_lens, dev(path), dev(acc))
    ref.keep(k, v, one.table, lens, path, acc)
    assert np.array_equal(f64(one.k)[None], k) and np.array_equal(f64(one.v)[None], v)


def test_keep_of_no_path(osd):
    import torch
    g = np.random.default_rng(6)
    lens = [5, 5, 5, 5, 5, 5, -1, 5, 5, 5]
    c = Cache(g, lens, 8, 2, 64, 4, "bf16", layers=2)
    path = np.tile(np.array([2, 3, 6, -1, -1, -1, -1, -1], np.int32), (10, 1))
    acc = np.array([3, -1, 8, 3, 3, 3, 3, 3, 0, 3], np.int32)
    path[3, :3] = [3, 2, 6]
    path[4, :3] = [0, 2, 6]
    path[5, :3] = [2, 6, 8]
    table = c.table.copy()
    table[7, 1] = 77       # the root's page
    table[9, 2] = -1       # a node's page
    k, v = f64(c.k).copy(), f64(c.v).copy()
    out = torch.full((10,), 99, dtype=torch.int32, device="cuda")
    new = osd.osd_cache_keep(c.k, c.v, dev(table), c.d_lens, dev(path), dev(acc), out=out)
    want = ref.keep(k, v, table, lens, path, acc)
    assert want.tolist() == [9, 5, 5, 5, 5, 5, -1, 5, 6, 5]
    assert new is out and new.cpu().numpy().tolist() == want.tolist()
    assert np.array_equal(f64(c.k), k) and np.array_equal(f64(c.v), v)


def test_append_and_keep_beyond_four_gigabytes(osd):
    import torch
    S, D, N = 256, 128, 6
    pages = 2 ** 31 // (S * D) + 5
    g = np.random.default_rng(8)
    k = torch.zeros(pages, 1, S, D, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    table, lens = dev(np.array([[pages - 1, pages - 2]], np.int32)), dev(np.array([254], np.int32))
    new = rows(g, 1, N, 1, D, "bf16")
    osd.osd_cache_append(new, new, k, v, table, lens)
    got = torch.cat([v[pages - 1, 0, 254:], v[pages - 2, 0, :4]])
    assert torch.equal(got, new[0, :, 0]) and float(v.abs().sum(dtype=torch.float64)) == float(new.abs().sum(dtype=torch.float64))
    path = dev(np.array([[2, 5, -1, -1, -1, -1]], np.int32))
    assert osd.osd_cache_keep(k, v, table, lens, path, dev(np.array([2], np.int32))).item() == 257
    assert torch.equal(v[pages - 1, 0, 255], new[0, 2, 0]) and torch.equal(k[pages - 2, 0, 0], new[0, 5, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_steps_of_speculative_decoding(osd, dtype):
    """Three steps: drafted trees appended, attended to, verified, the accepted
    paths kept.  Every call against the reference; the cache afterwards holds what
    appending the emitted tokens one by one gives."""
    import torch
    g = np.random.default_rng(9)
    B, N, Hq, H, D, S, V, layers = 3, 10, 4, 2, 64, 8, 50, 2
    lens0 = [5, 0, 30]
    c = Cache(g, [n + 3 * N for n in lens0], N, H, D, S, dtype, layers=layers)
    lens = dev(np.array(lens0, np.int32))
    turn, dt = rotation(80, D), torch_dtype(dtype)
    plain = [c.k.clone(), c.v.clone()]
    for step in range(3):
        now = lens.cpu().numpy()
        parent = trees(g, B, N)
        tokens = g.integers(0, V, (B, N)).astype(np.int32)
        new = [[rows(g, B, N, h, D, dtype) for h in (Hq, H, H)] for _ in range(layers)]
        for l, (q, k, v) in enumerate(new):
            kc, vc = f64(c.k[l]), f64(c.v[l])
            qr = osd.osd_cache_append(k, v, c.k[l], c.v[l], c.d_table, lens, q=q, rotation=dev(turn), parent=dev(parent))
            out, kc, vc = ref.append(f64(q), f64(k), f64(v), kc, vc, c.table, now, turn.astype(np.float64), False, parent)
            check_rotated(qr, out, pair_sizes(f64(q), D, False), dtype, "q")
            o = osd.osd_tree_attention(qr, c.k[l], c.v[l], c.d_table, lens, dev(parent))
            want, mass, reach = ref.attention(f64(qr), f64(c.k[l]), f64(c.v[l]), c.table, now, D ** -0.5, parent)
            check_attention(o, want, mass, reach, int(now.max()) + N, dtype)
        logits = dev(g.normal(0, 1, (B, N, V)).astype(np.float32), dt)
        draft = logits + 0.1 * torch.randn_like(logits)
        u, ur = dev(g.random((B, N)).astype(np.float32)), dev(g.random(B).astype(np.float32))
        acc, toks, path = osd.osd_verify_tree(logits, draft, dev(parent), dev(tokens), u, ur, 1.0)
        lens = osd.osd_cache_keep(c.k, c.v, c.d_table, lens, path, acc)
        acc, path = acc.cpu().numpy(), path.cpu().numpy()
        assert (acc >= 0).all() and np.array_equal(lens.cpu().numpy(), now + 1 + acc)
        # The same tokens appended as chains to the other cache.
        for l, (q, k, v) in enumerate(new):
            for b in range(B):
                nodes = [0] + path[b, :acc[b]].tolist()
                osd.osd_cache_append(k[b:b + 1, nodes].contiguous(), v[b:b + 1, nodes].contiguous(), plain[0][l], plain[1][l],
                                     c.d_table[b:b + 1].contiguous(), dev(now[b:b + 1]), rotation=dev(turn))
    for b in range(B):
        for j in range(int(lens[b])):
            p, s = c.row(b, j)
            assert torch.equal(c.k[:, p, :, s], plain[0][:, p, :, s]) and torch.equal(c.v[:, p, :, s], plain[1][:, p, :, s])
