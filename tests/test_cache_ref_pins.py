"""Pins of the paged cache's reference (oracle/cache_ref.py): facts that the
definitions fix, on the CPU."""
import numpy as np
import pytest

from oracle import cache_ref as ref


def cache(g, P, H, S, D):
    return g.normal(size=(P, H, S, D)), g.normal(size=(P, H, S, D))


def test_lines_are_the_paths_from_the_root():
    assert ref.lines([0, 0, 0, 1, 3, 2], 6) == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0, 2, 5]]
    assert ref.lines(None, 3) == [[0], [0, 1], [0, 1, 2]]
    assert ref.lines([7, 0, 2], 3) is None and ref.lines([0, -1], 2) is None and ref.lines([9], 1) == [[0]]


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_is_complex_multiplication(pairs):
    g = np.random.default_rng(0)
    R, D = 6, 10
    angle = g.uniform(0, 6, R // 2)
    x = g.normal(size=(3, D))
    y = ref.rotate(x, np.concatenate([np.cos(angle), np.sin(angle)]), pairs)
    z = x[:, 0:R:2] + 1j * x[:, 1:R:2] if pairs else x[:, :3] + 1j * x[:, 3:6]
    w = z * np.exp(1j * angle)
    got = y[:, 0:R:2] + 1j * y[:, 1:R:2] if pairs else y[:, :3] + 1j * y[:, 3:6]
    assert np.allclose(got, w, atol=1e-14) and np.array_equal(y[:, R:], x[:, R:])


def test_scores_of_rotated_rows_depend_on_the_distance_alone():
    g = np.random.default_rng(1)
    D = 8
    pos = np.arange(40)[:, None] * 100.0 ** (-np.arange(D // 2) / (D // 2))
    turn = np.concatenate([np.cos(pos), np.sin(pos)], 1)
    q, k = g.normal(size=(1, D)), g.normal(size=(1, D))
    s = [(ref.rotate(q, turn[p + 7], False) @ ref.rotate(k, turn[p], False).T).item() for p in (0, 3, 30)]
    assert np.allclose(s, s[0], atol=1e-12)


def test_a_node_sees_what_a_chain_of_its_ancestors_sees():
    g = np.random.default_rng(2)
    S, D, c = 4, 6, 9
    kc, vc = cache(g, 5, 2, S, D)
    table = np.array([[3, 0, 4, 1, 2]])
    parent = np.array([[0, 0, 0, 2, 1, 3]])
    q = g.normal(size=(1, 6, 4, D))
    out, mass, reach = ref.attention(q, kc, vc, table, [c], 0.4, parent)
    for i, line in enumerate(ref.lines(parent[0], 6)):
        for hq in range(4):
            h = hq // 2
            rows = [(table[0, j // S], j % S) for j in list(range(c)) + [c + a for a in line]]
            x = np.array([0.4 * kc[p, h, s] @ q[0, i, hq] for p, s in rows])
            w = np.exp(x) / np.exp(x).sum()
            want = sum(wj * vc[p, h, s] for wj, (p, s) in zip(w, rows))
            assert np.allclose(out[0, i, hq], want, atol=1e-13)
    assert (mass >= np.abs(out) - 1e-12).all() and (reach > 0).all()
    # parent None is the chain
    chain = np.array([[0, 0, 1, 2, 3, 4]])
    assert np.array_equal(ref.attention(q, kc, vc, table, [c], 0.4)[0], ref.attention(q, kc, vc, table, [c], 0.4, chain)[0])


def test_padding_and_invalid_sequences():
    g = np.random.default_rng(3)
    kc, vc = cache(g, 4, 1, 4, 8)
    table = np.array([[0, 1], [2, 9], [2, 3], [2, 3]])
    q = g.normal(size=(4, 2, 1, 8))
    out = ref.attention(q, kc, vc, table, [3, 3, -1, 2], 1.0, new_len=[1, 2, 2, 3])[0]
    assert np.isfinite(out[0, 0]).all() and (out[0, 1] == 0).all()
    assert np.isnan(out[1]).all() and (out[2] == 0).all() and np.isnan(out[3]).all()


def test_step_of_append_attention_and_keep():
    """Appending an accepted path after keep gives the cache that appending
    its tokens one by one gives."""
    g = np.random.default_rng(4)
    H, S, D, N, c = 2, 4, 8, 6, 5
    kc, vc = cache(g, 4, H, S, D)
    table = np.array([[2, 0, 3, 1]])
    pos = np.arange(20)[:, None] * 10.0 ** (-np.arange(D // 2) / (D // 2))
    turn = np.concatenate([np.cos(pos), np.sin(pos)], 1)
    k, v, q = (g.normal(size=(1, N, H, D)) for _ in range(3))
    parent = np.array([[0, 0, 0, 2, 1, 3]])
    _, k1, v1 = ref.append(q, k, v, kc, vc, table, [c], turn, False, parent)
    path = np.array([[2, 3, 5, -1, -1, -1]])
    k1, v1 = k1[None], v1[None]
    assert ref.keep(k1, v1, table, [c], path, [3]).tolist() == [c + 4]
    k2, v2 = kc, vc
    for i, node in enumerate([0, 2, 3, 5]):
        _, k2, v2 = ref.append(q[:, node:node + 1], k[:, node:node + 1], v[:, node:node + 1], k2, v2, table, [c + i], turn)
    for j in range(c + 4):
        p, s = table[0, j // S], j % S
        assert np.allclose(k1[0, p, :, s], k2[p, :, s], atol=1e-14) and np.array_equal(v1[0, p, :, s], v2[p, :, s])


@pytest.mark.parametrize("path,accepted", [([[2, 1, 3]], [3]), ([[0, 1, 2]], [1]), ([[1, 2, 3]], [3]), ([[1, 1, 2]], [2]),
                                           ([[1, 2, 2]], [-1])])
def test_keep_of_no_path_moves_nothing(path, accepted):
    g = np.random.default_rng(5)
    kc, vc = (x[None] for x in cache(g, 2, 1, 4, 8))
    before = kc.copy()
    assert ref.keep(kc, vc, np.array([[0, 1]]), [2], np.array(path), accepted).tolist() == [2]
    assert np.array_equal(kc, before)
