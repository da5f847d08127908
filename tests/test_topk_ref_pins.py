"""What pins the reference of the records of top logits (oracle/topk_ref.py):
brute force, the whole-row oracle at k = V, finite differences, and the
exactness of verification with a truncated draft."""
import numpy as np
import pytest

from oracle import ref, topk_ref
from tests._topk_helpers import as_dtype, rows, uniforms


def test_topk_by_brute_force():
    x = rows("ties", 5, 40, 1)
    got = topk_ref.topk(x, 7, 0.5, uniforms(5, 2))
    for n in range(5):
        want = sorted(range(40), key=lambda j: (-x[n, j], j))[:7]
        assert got["ids"][n].tolist() == want
        out = [j for j in range(40) if j not in want]
        mass = sum(np.exp((float(x[n, j]) - float(x[n, want[0]])) / 0.5) for j in out)
        assert abs(got["rest"][n] - np.log(mass)) < 1e-12
        assert got["tokens"][n] in want


def test_topk_edges():
    x = np.array([[0.0, -0.0, -np.inf, 1.0], [-np.inf] * 4, [np.nan, 1, 2, 3], [np.inf, 1, 2, 3]], np.float32)
    got = topk_ref.topk(x, 4, 1.0, np.zeros(4, np.float32))
    assert got["ids"].tolist() == [[3, 0, 1, -1], [-1] * 4, [-1] * 4, [-1] * 4]
    assert got["rest"].tolist() == [-np.inf] * 4
    assert got["tokens"].tolist() == [3, -1, -1, -1]


def test_draw_follows_the_record():
    """Stratified uniforms give M pi_r +- 1 draws of each slot."""
    M = 4000
    x = np.repeat(rows("normal", 1, 30, 3), M, 0)
    got = topk_ref.topk(x, 5, 0.8, ((np.arange(M) + 0.5) / M).astype(np.float32))
    pi = topk_ref.softmax(got["top"][0] / 0.8)
    for r in range(5):
        assert abs((got["tokens"] == got["ids"][0, r]).sum() - M * pi[r]) <= 1.01


@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_whole_row_record_is_the_whole_row_divergence(kind, dtype):
    V, N, tau = 33, 4, 0.75
    t, s = as_dtype(rows("normal", N, V, 4), dtype), as_dtype(rows("normal", N, V, 5), dtype)
    rec = topk_ref.topk(t, V, tau)
    top = np.take_along_axis(t, rec["ids"].astype(np.int64), 1)
    assert (rec["rest"] == -np.inf).all()
    loss, D, g = topk_ref.distill(rec["ids"], top, rec["rest"], s, kind, 0.3, tau)
    want = ref.distill(t.reshape(N, 1, V), s.reshape(N, 1, V), kind, 0.3, tau)
    assert np.allclose(loss, [want["loss_mean"], want["loss_sum"]], rtol=1e-12)
    assert np.allclose(D, want["row_loss"].reshape(-1), rtol=1e-10, atol=1e-14)
    assert np.allclose(g, want["grad"].reshape(N, V), rtol=1e-9, atol=1e-14)


@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("with_rest", [True, False])
def test_gradient_by_differences(kind, with_rest):
    if kind == "rkl" and not with_rest:
        pytest.skip("infinite")
    V, k, tau, beta, h = 12, 4, 1.3, 0.4, 1e-4
    t = rows("normal", 1, V, 6)
    s = rows("normal", 1, V, 7).astype(np.float64)
    rec = topk_ref.topk(t, k, tau)
    top = np.take_along_axis(t, rec["ids"].astype(np.int64), 1)
    rest = rec["rest"] if with_rest else None
    f = lambda z: topk_ref.distill(rec["ids"], top, rest, z, kind, beta, tau)
    _, D, g = f(s)
    assert D[0] > 0 and abs(g.sum()) < 1e-12
    for j in range(V):
        e = np.zeros_like(s)
        e[0, j] = h
        assert abs((f(s + e)[1][0] - f(s - e)[1][0]) / (2 * h) - g[0, j]) < 1e-6


def test_coarse_divergence_is_at_most_the_whole_rows():
    """Summing tokens into a bucket never raises a divergence."""
    V, N = 50, 6
    t, s = rows("normal", N, V, 8), rows("normal", N, V, 9)
    for kind in ("fkl", "rkl", "jsd"):
        last = np.inf
        whole = ref.distill(t.reshape(N, 1, V), s.reshape(N, 1, V), kind, 0.5, 1.0)["row_loss"].reshape(-1)
        for k in (V, 30, 10, 1):
            rec = topk_ref.topk(t, k, 1.0)
            top = np.take_along_axis(t, rec["ids"].astype(np.int64), 1)
            D = topk_ref.distill(rec["ids"], top, rec["rest"], s, kind, 0.5, 1.0)[1]
            assert (D <= np.minimum(last, whole) + 1e-12).all()
            last = D


def test_closed_form_of_two_buckets():
    """k = 1: Bernoulli divergences."""
    t, s = np.array([[2.0, 0.0, 0.0]], np.float32), np.array([[0.5, 1.0, -1.0]], np.float32)
    rec = topk_ref.topk(t, 1, 1.0)
    p = np.exp(2.0) / (np.exp(2.0) + 2)
    q = np.exp(0.5) / (np.exp(0.5) + np.exp(1.0) + np.exp(-1.0))
    D = topk_ref.distill(rec["ids"], np.array([[2.0]], np.float32), rec["rest"], s, "fkl", 0.5, 1.0)[1][0]
    assert abs(D - (p * np.log(p / q) + (1 - p) * np.log((1 - p) / (1 - q)))) < 1e-12


@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_jsd_endpoints_are_zero(beta):
    t, s = rows("normal", 2, 20, 10), rows("normal", 2, 20, 11)
    rec = topk_ref.topk(t, 5, 1.0)
    top = np.take_along_axis(t, rec["ids"].astype(np.int64), 1)
    for rest in (rec["rest"], None):
        loss, D, g = topk_ref.distill(rec["ids"], top, rest, s, "jsd", beta, 1.0)
        assert (D == 0).all() and (g == 0).all() and (loss == 0).all()


def test_bad_records_and_rows_give_nan_masked_ones_zero():
    V, k = 10, 3
    s = rows("normal", 7, V, 12)
    ids = np.tile(np.array([1, 2, 3], np.int32), (7, 1))
    top = np.tile(np.array([3.0, 2.0, 1.0], np.float32), (7, 1))
    ids[1] = [1, 2, 1]
    ids[2, 1] = V
    top[3, 2] = np.nan
    ids[4], top[4] = -1, -np.inf
    s[5, 0] = np.nan
    mask = np.ones(7, np.uint8)
    mask[6] = 0
    _, D, g = topk_ref.distill(ids, top, np.zeros(7), s, "fkl", 0.5, 1.0, mask)
    assert np.isfinite(D[0]) and np.isnan(D[1:6]).all() and D[6] == 0 and (g[6] == 0).all()
    assert np.isnan(g[1:6]).all() and np.isfinite(g[0]).all()


@pytest.mark.parametrize("ragged", [False, True])
def test_verify_whole_row_record_is_osd_verify(ragged):
    B, K, V, T = 40, 4, 25, 0.75
    t, d = rows("normal", B * (K + 1), V, 13).reshape(B, K + 1, V), rows("normal", B * K, V, 14).reshape(B, K, V)
    rec = topk_ref.topk(d.reshape(-1, V), V, T, uniforms(B * K, 15))
    ids = rec["ids"].reshape(B, K, V)
    top = np.take_along_axis(d, ids.astype(np.int64), 2)
    y = rec["tokens"].reshape(B, K)
    ua, ur = uniforms((B, K), 16), uniforms(B, 17)
    dl = (np.arange(B) % K + 1).astype(np.int32) if ragged else None
    acc, out, rmask, _ = topk_ref.verify(t, ids, top, y, ua, ur, T, dl)
    want = ref.verify(t, d, y, ua, ur, T, draft_len=dl)
    assert np.array_equal(acc, want["accepted_len"]) and np.array_equal(out, want["out_tokens"])
    assert np.array_equal(rmask, want["reject_mask"])


def test_emitted_token_follows_the_target_although_the_draft_is_truncated():
    """K = 1: sum over proposals of q(y) times the outcome over a grid of
    uniforms gives p."""
    V, k, M = 6, 2, 60
    t, d = rows("normal", 2, V, 18).reshape(1, 2, V) / 2, rows("normal", 1, V, 19) / 2
    rec = topk_ref.topk(d, k, 1.0)
    q = topk_ref.softmax(rec["top"][0])
    grid = ((np.arange(M) + 0.5) / M).astype(np.float32)
    B = M * M
    ua, ur = np.repeat(grid, M).reshape(B, 1), np.tile(grid, M)
    freq = np.zeros(V)
    for slot in range(k):
        y = np.full((B, 1), rec["ids"][0, slot], np.int32)
        out = topk_ref.verify(np.repeat(t, B, 0), np.repeat(rec["ids"][None], B, 0),
                              np.repeat(rec["top"][None].astype(np.float32), B, 0), y, ua, ur, 1.0)[1]
        freq += q[slot] * np.bincount(out[:, 0], minlength=V) / B
    assert np.abs(freq - topk_ref.softmax(t[0, 0].astype(np.float64))).max() < 2.0 / M


def test_verify_invalid_sequences():
    B, K, V = 7, 2, 8
    t = rows("normal", B * 3, V, 20).reshape(B, 3, V)
    ids = np.tile(np.array([1, 2, 3], np.int32), (B, K, 1))
    top = np.tile(np.array([3.0, 2.0, 1.0], np.float32), (B, K, 1))
    y = np.ones((B, K), np.int32)
    ua, ur = np.zeros((B, K), np.float32), np.full(B, 0.5, np.float32)  # all tests pass
    dl = np.full(B, K, np.int32)
    ids[1, 1] = [1, 1, 2]
    y[2, 1] = V
    dl[3] = 0
    t[4, 2] = -np.inf
    top[5, 0, 1] = np.inf
    ids[6, 1] = -1
    acc = topk_ref.verify(t, ids, top, y, ua, ur, 1.0, dl)[0]
    assert acc.tolist() == [2, -1, -1, -1, -1, -1, -1]
    ua[1, 0] = ua[6, 0] = 0.999999  # rejected before the bad record is tested
    top[:, 0, 0] = 60.0
    acc = topk_ref.verify(t, ids, top, y, ua, ur, 1.0, dl)[0]
    assert acc[1] == 0 and acc[6] == 0


@pytest.mark.parametrize("gap", [0.0, 600.0, 740.0, 800.0, 1.0e4])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
def test_gradient_of_others_far_below_is_autograd(kind, gap):
    """Against torch's derivative of the definition in logarithms, in fp64, where
    the others' mass has left its range."""
    import torch
    V, k, tau, beta = 40, 6, 1.3, 0.4
    t = rows("normal", 1, V, 30)
    rec = topk_ref.topk(t, k, tau)
    ids = rec["ids"][0].astype(np.int64)
    top = np.take_along_axis(t, rec["ids"].astype(np.int64), 1)
    s = rows("normal", 1, V, 31).astype(np.float64) - gap
    s[0, ids] += gap
    x = torch.tensor(s[0], requires_grad=True)
    lq = torch.log_softmax(x / tau, 0)
    out = np.setdiff1d(np.arange(V), ids)
    lb = torch.cat([lq[ids], torch.logsumexp(lq[out], 0).view(1)])
    lt = np.append((rec["top"][0] - rec["top"][0, 0]) / tau, np.float32(rec["rest"][0]))
    lp = torch.log_softmax(torch.tensor(lt), 0)
    if kind == "fkl":
        D = (lp.exp() * (lp - lb)).sum()
    elif kind == "rkl":
        D = (lb.exp() * (lb - lp)).sum()
    else:
        lm = torch.logaddexp(lp + np.log(beta), lb + np.log(1 - beta))
        D = beta * (lp.exp() * (lp - lm)).sum() + (1 - beta) * (lb.exp() * (lb - lm)).sum()
    D.backward()
    _, rl, g = topk_ref.distill(rec["ids"], top, rec["rest"].astype(np.float32), s, kind, beta, tau)
    assert abs(rl[0] - D.item()) < 1e-12 * max(1.0, D.item())
    assert np.abs(g[0] - x.grad.numpy()).max() < 1e-12
    assert abs(g.sum()) < 1e-12


@pytest.mark.parametrize("T", [1.0, 0.02, 0.001])
def test_rest_far_below_the_record(T):
    """Against torch's logsumexp; where exp of the difference is 0 in fp64 too."""
    import torch
    x = rows("normal", 5, 300, 40)
    x[1, 7] += 900.0
    x[2, :10] += 5.0e3
    rec = topk_ref.topk(x, 10, T)
    for n in range(5):
        out = np.delete(x[n].astype(np.float64), rec["ids"][n])
        want = torch.logsumexp(torch.tensor((out - rec["top"][n, 0]) / T), 0).item()
        assert abs(rec["rest"][n] - want) < 1e-12 * max(1.0, abs(want))
