"""osd_tree_attention where values are not finite: a row that sees one gets exactly
that, whatever its key's place in a tile, and however the work is divided."""
import numpy as np
import pytest

from oracle import cache_ref as ref
from tests._cache_helpers import E, HALF, Cache, check_attention, dev, f64, torch_dtype, trees

pytestmark = pytest.mark.gpu

WHAT = {"nan": float("nan"), "inf": float("inf"), "-inf": -float("inf")}


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


def queries(g, B, N, Hq, D, dtype):
    return dev(g.normal(0, 1, (B, N, Hq, D)).astype(np.float32), torch_dtype(dtype))


@pytest.mark.parametrize("N,G", [(3, 4), (5, 4), (32, 4), (64, 4)])
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cut", [False, True])
def test_the_context_last_tokens(osd, cut, dtype, D, N, G):
    """Three values of each of the last 64 tokens of the context in turn, contexts of all
    residues of a stage, units in a row (few of them shared) or cut apart: all nodes see
    them, in three values of one kv head's rows, and nothing else changes but by rounding.

    (A sum that is not finite has a workgroup's keys taken again, relative to another score, so
    bits of the other values may change.  Both outputs are off by at most (2 r + n E + 2^-15 + 2^-22) sum p |v| and
    half a step of themselves, r and the probabilities' part as in _cache_helpers and
    test_attention_rounding_gpu; sum p |v| <= max |v|, and a score's sum |q||k| is at most the product of the
    norms.  They differ by at most twice that, and 2.02 half steps, as the one is within 2^-7 of the other.)"""
    import torch
    g = np.random.default_rng(D + N)
    H = 1 if cut else 12
    head, columns = H - 1, {5: "inf", D // 2: "-inf", D - 3: "nan"}
    at = sorted(columns)
    values = torch.tensor([WHAT[columns[x]] for x in at], device="cuda")
    for lens in (np.arange(130, 194).reshape(-1, 4) if cut else np.arange(66, 130).reshape(1, -1)).tolist():
        B = len(lens)
        c = Cache(g, lens, N, H, D, 16, dtype)
        q, parent = queries(g, B, N, G * H, D, dtype), dev(trees(g, B, N))
        clean = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
        assert torch.isfinite(clean).all()
        n, size = max(lens) + N, lambda t: float(t.float().norm(dim=-1).max())
        r = ((D + 5) * D ** -0.5 * size(q) * size(c.k) + 2 + n + 3 * n / 32 + 8) * E
        apart = 2.02 * (2 * r + n * E + (2.0 ** -15 + 2.0 ** -22 if dtype == "bf16" else 0.0)) * float(c.v.float().abs().max())
        tol = apart + 2.02 * HALF[dtype] * clean.float().abs()
        wrong = torch.zeros((), device="cuda", dtype=torch.bool)
        for back in range(1, 65):
            j = c.d_lens.long() - back
            page, slot = c.d_table.long().gather(1, (j // 16)[:, None])[:, 0], j % 16
            held = c.v[page, head, slot].clone()
            row = held.clone()
            row[:, at] = values.to(row.dtype)
            c.v[page, head, slot] = row
            got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, parent)
            c.v[page, head, slot] = held
            hit = got[:, :, head * G:].float()[..., at]
            wrong |= ~torch.where(values.isnan(), hit.isnan(), hit == values).all()
            got[:, :, head * G:, at] = clean[:, :, head * G:, at]
            wrong |= ~((got.float() - clean.float()).abs() <= tol).all()
            if back % 16 == 0:
                assert not wrong, (lens[0], back)


@pytest.mark.parametrize("N,G,H", [(16, 1, 1), (4, 4, 2), (64, 1, 1), (32, 4, 1), (64, 4, 1), (33, 2, 140)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("D", [64, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nodes_on_both_sides_of_a_border(osd, dtype, D, tree, N, G, H):
    """Nodes of which some lie in one stage and some in the next, which other
    workgroups may have: a row gets what it sees of both, and of none of them."""
    g = np.random.default_rng(N + D)
    for n in range(65, 260, 27 if H < 100 else 130):
        c = Cache(g, [n, 40], N, H, D, 16, dtype)
        q, parent = queries(g, 2, N, G * H, D, dtype), trees(g, 2, N) if tree else None
        early, late = int(g.integers(0, N // 2)), int(g.integers(N // 2, N))
        for node, values in ((early, {1: "inf", 3: "inf", 4: "nan", 6: "-inf"}), (late, {2: "-inf", 3: "inf", 5: "nan", 6: "inf"})):
            page, slot = c.row(0, n + node)
            for column, what in values.items():
                c.v[page, :, slot, column] = WHAT[what]
        got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, None if parent is None else dev(parent))
        want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, [n, 40], D ** -0.5, parent)
        check_attention(got, want, mass, reach, n + N, dtype, f"{n} {early} {late}")


@pytest.mark.parametrize("N,G,D", [(1, 4, 128), (4, 4, 64), (3, 2, 256), (16, 4, 128), (32, 4, 64), (64, 4, 128), (40, 2, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_values(osd, dtype, N, G, D):
    """Values of 2^100 whose weights relative to a step's first keys reach 2^28.9: outputs are finite."""
    import torch
    g = np.random.default_rng(71)
    H, B = 4, 24 if N < 5 else 8
    lens = [int(x) for x in g.integers(400, 1500, B)]
    c = Cache(g, lens, N, H, D, 16, dtype)
    c.v.mul_(2.0 ** 100)
    c.k.zero_()
    q = torch.zeros(B, N, G * H, D, device="cuda", dtype=torch_dtype(dtype))
    q[..., 0] = 4.0
    for b, n in enumerate(lens):
        high = torch.from_numpy(g.random((n + N + 31) // 32) < 0.5).repeat_interleave(32)[:n + N].cuda()
        j = torch.arange(n + N, device="cuda")
        page = c.d_table[b].long()[j // 16]
        c.k[page, :, j % 16, 0] = torch.where(high, 5.0, 0.0).to(c.k.dtype)[:, None]
    got = osd.osd_tree_attention(q, c.k, c.v, c.d_table, c.d_lens, scale=1.0)
    want, mass, reach = ref.attention(f64(q), f64(c.k), f64(c.v), c.table, lens, 1.0)
    assert np.isfinite(want).all()
    check_attention(got, want, mass, reach, max(lens) + N, dtype)
