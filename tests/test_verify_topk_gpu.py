"""osd_verify_topk against the 64-bit reference: every output exactly (a
sequence with a decision within 1e-9 of a border is counted and left out), and
a speculative step that makes, draws from, verifies and distils records."""
import numpy as np
import pytest

from oracle import topk_ref
from tests._helpers import to_device
from tests._topk_helpers import as_dtype, lowest, rows, uniforms
from tests.test_topk_gpu import host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


def inputs(B, K, V, k, dtype, T, seed, noise=1.0, kind="normal"):
    t = rows(kind, B * (K + 1), V, seed, dtype).reshape(B, K + 1, V)
    with np.errstate(over="ignore", invalid="ignore"):
        d = (rows("normal", B * K, V, seed + 1) / 3 * noise).reshape(B, K, V)
        d = d + np.where(np.abs(t[:, :K]) < 1e4, t[:, :K], 0)
    t, d = as_dtype(t, dtype), as_dtype(d, dtype)
    rec = topk_ref.topk(d.reshape(B * K, V), k, T, uniforms(B * K, seed + 2))
    ids = rec["ids"]
    top = np.take_along_axis(d.reshape(B * K, V), ids.astype(np.int64), 1)
    return dict(t=t, ids=ids.reshape(B, K, k), top=top.reshape(B, K, k), y=rec["tokens"].reshape(B, K),
                ua=uniforms((B, K), seed + 3), ur=uniforms(B, seed + 4))


def call(osd, x, T, dl=None):
    return osd.osd_verify_topk(*(to_device(x[n]) for n in ("t", "ids", "top", "y", "ua", "ur")), T,
                               draft_len=to_device(dl))


def check(got, x, T, dl, label):
    acc, toks, rmask = (host(t) for t in got)
    wa, wt, wm, margin = topk_ref.verify(x["t"], x["ids"], x["top"], x["y"], x["ua"], x["ur"], T, dl)
    sure = margin > 1e-9
    bad = (acc != wa) | (toks != wt).any(1) | (rmask != wm).any(1)
    bad &= sure
    assert not bad.any(), (f"{label}: {bad.sum()} sequences, first {np.argwhere(bad)[0]}: {acc[bad][0]} "
                           f"{toks[bad][0]} for {wa[bad][0]} {wt[bad][0]}")
    return int((~sure).sum())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(1, 1), (2, 1), (7, 7), (9, 4), (100, 64), (255, 3), (1001, 65), (2048, 256),
                                 (2049, 16), (4099, 1), (8192, 100), (20011, 33), (32000, 64), (32771, 255)])
def test_shapes(osd, V, k, dtype):
    B, K, T = 7, 3, 0.75
    x = inputs(B, K, V, k, dtype, T, V)
    assert check(call(osd, x, T), x, T, None, f"V={V} k={k} {dtype}") <= 1


@pytest.mark.parametrize("V,k,dtype", [(65536, 100, "f32"), (50257, 20, "f32"), (131072, 256, "bf16"),
                                       (128256, 64, "bf16"), (100003, 17, "bf16")])
def test_long_rows(osd, V, k, dtype):
    B, K, T = 2, 2, 1.0
    x = inputs(B, K, V, k, dtype, T, V)
    check(call(osd, x, T), x, T, None, f"V={V} k={k} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 2, 5, 16])
@pytest.mark.parametrize("noise", [0.05, 3.0])
def test_lengths_and_acceptance(osd, K, noise, dtype):
    """Ragged and out-of-range lengths; drafts near the target and far off."""
    B, V, k, T = 60, 1003, 50, 1.0
    x = inputs(B, K, V, k, dtype, T, 100 + K, noise)
    dl = (np.arange(B) % (K + 2)).astype(np.int32)
    left = check(call(osd, x, T, dl), x, T, dl, f"K={K} ragged") + check(call(osd, x, T), x, T, None, f"K={K}")
    assert left <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["ties", "equal", "lowest", "masked", "masked_lowest", "ascending", "block", "peak",
                                  "wide", "bad"])
@pytest.mark.parametrize("V", [777, 40003])
def test_target_kinds(osd, kind, V, dtype):
    B, K, k, T = 6, 3, 40, 1.0
    x = inputs(B, K, V, k, dtype, T, 7, kind=kind)
    x["ur"][0] = 0.0
    x["ur"][1] = np.float32(1 - 2.0 ** -24)
    x["ua"][2] = 0.0
    x["ua"][3] = np.float32(1 - 2.0 ** -24)
    check(call(osd, x, T), x, T, None, f"{kind} V={V} {dtype}")


def test_first_and_last_tokens(osd):
    """u = 0 draws the first token with mass, the largest u the last ones; the
    residual of a draft with all of the target's mass."""
    B, K, V, k, T = 4, 1, 5000, 8, 1.0
    t = np.full((B, 2, V), -np.inf, np.float32)
    t[:, :, [3, 2500, 4990]] = np.array([0.0, 0.5, 1.0], np.float32)
    ids = np.full((B, K, k), -1, np.int32)
    top = np.full((B, K, k), -np.inf, np.float32)
    ids[:, :, 0], top[:, :, 0] = 4990, 1.0
    x = dict(t=t, ids=ids, top=top, y=np.full((B, K), 4990, np.int32),
             ua=np.full((B, K), 1 - 2.0 ** -24, np.float32), ur=np.array([0, 1 - 2.0 ** -24, 0.3, 0.6], np.float32))
    acc, toks, _ = (host(o) for o in call(osd, x, T))
    assert acc.tolist() == [0] * 4 and toks[:2, 0].tolist() == [3, 2500]
    check(call(osd, x, T), x, T, None, "sparse")
    x["ua"][:] = 0.0
    check(call(osd, x, T), x, T, None, "bonus")


def test_bad_records_tokens_and_rows(osd):
    B, K, V, k, T = 12, 3, 3000, 30, 1.0
    for accept in (0.0, 1 - 2.0 ** -24):
        x = inputs(B, K, V, k, "f32", T, 55)
        x["ua"][:] = accept
        x["ids"][0, 0, 3] = x["ids"][0, 0, 9]
        x["ids"][1, 2, 3] = V
        x["ids"][2, 1, 3] = -5
        x["top"][3, 1, 0] = np.nan
        x["top"][4, 1, 0] = np.inf
        x["ids"][5, 2] = -1
        x["y"][6, 2] = V
        x["y"][7, 0] = -1
        x["t"][8, 3] = -np.inf
        x["t"][9, 1, 5] = np.nan
        x["ids"][10, 0, 4:] = -1  # a short record is one
        check(call(osd, x, T), x, T, None, f"bad accept={accept}")


def test_proposal_outside_its_record(osd):
    x = inputs(5, 2, 1000, 10, "f32", 1.0, 66)
    x["y"][:, 0] = [j for j in range(1000) if j not in x["ids"][:, 0]][:5]
    acc = host(call(osd, x, 1.0)[0])
    assert (acc >= 1).all()
    check(call(osd, x, 1.0), x, 1.0, None, "outside")


@pytest.mark.parametrize("B", [1, 64, 400])
def test_batches_repeat(osd, B):
    """Calls of several sizes in a row on one workspace give equal bits."""
    import torch
    K, V, k, T = 4, 8001, 64, 1.0
    x = inputs(min(B, 16), K, V, k, "bf16", T, 77)
    x = {n: np.concatenate([a] * (-(-B // len(a))))[:B] for n, a in x.items()}
    a = call(osd, x, T)
    first = {n: v[:16] for n, v in x.items()}
    check([t[:16] for t in a], first, T, None, f"B={B}")
    b = call(osd, first, T)
    assert all(torch.equal(p[:min(B, 16)], q) for p, q in zip(a, b))
    c = call(osd, x, T)
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_whole_row_record_is_osd_verify(osd):
    """k = V: osd_verify's outcome (its own fp32 margin, 1e-6, left out)."""
    B, K, V, T = 50, 3, 200, 1.0
    g = rows("normal", B * K, V, 88)
    t, d = rows("normal", B * (K + 1), V, 89).reshape(B, K + 1, V), g.reshape(B, K, V)
    rec = topk_ref.topk(g, V, T, uniforms(B * K, 90))
    x = dict(t=t, ids=rec["ids"].reshape(B, K, V), top=rec["top"].astype(np.float32).reshape(B, K, V),
             y=rec["tokens"].reshape(B, K), ua=uniforms((B, K), 91), ur=uniforms(B, 92))
    a = [host(o) for o in call(osd, x, T)]
    b = [host(o) for o in osd.osd_verify(to_device(t), to_device(d), to_device(x["y"]), to_device(x["ua"]),
                                         to_device(x["ur"]), T)]
    margin = topk_ref.verify(t, x["ids"], x["top"], x["y"], x["ua"], x["ur"], T)[3]
    sure = margin > 1e-6
    assert sure.sum() > 45
    assert all(np.array_equal(p[sure], q[sure]) for p, q in zip(a, b))


def test_guard_bands_and_workspace(osd):
    import ctypes
    import torch
    from paper_2310_07177_amd import binding
    for B, K, V, k in [(1, 1, 5, 3), (7, 3, 1001, 20), (3, 16, 4099, 64)]:
        x = inputs(B, K, V, k, "bf16", 1.0, 99)
        d = [to_device(x[n]) for n in ("t", "ids", "top", "y", "ua", "ur")]
        sizes = [B * 4, B * (K + 1) * 4, B * K]
        bufs = [torch.full((z + 8192,), 0x5A, dtype=torch.uint8, device="cuda") for z in sizes]
        ws = torch.zeros(osd.lib().osd_verify_topk_workspace_bytes(B, K) + 4096, dtype=torch.uint8, device="cuda")
        ws[-4096:] = 0x5A
        p = lambda t, o=0: ctypes.c_void_p(t.data_ptr() + o)
        st = osd.lib().osd_verify_topk(p(d[0]), p(d[1]), p(d[2]), k, binding.OSD_BF16, B, K, V, p(d[3]), None, p(d[4]),
                                       p(d[5]), 1.0, *(p(b, 4096) for b in bufs), p(ws), ws.numel() - 4096, None)
        assert st == 0
        torch.cuda.synchronize()
        assert (ws[-4096:] == 0x5A).all()
        for b, z in zip(bufs, sizes):
            assert (b[:4096] == 0x5A).all() and (b[4096 + z:] == 0x5A).all()


def test_graph(osd):
    import torch
    B, K, V, k, T = 6, 4, 9001, 64, 1.0
    xs = [inputs(B, K, V, k, "bf16", T, 200 + i) for i in range(3)]
    names = ("t", "ids", "top", "y", "ua", "ur")
    held = [to_device(xs[0][n]).clone() for n in names]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        osd.osd_verify_topk(*held, T)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = osd.osd_verify_topk(*held, T)
    for i in (1, 2, 0, 1):
        for h, n in zip(held, names):
            h.copy_(to_device(xs[i][n]))
        eager = osd.osd_verify_topk(*held, T)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        check(out, xs[i], T, None, f"replay {i}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_speculative_step_on_records(osd, dtype):
    """A step as it is used: K proposals drawn from the draft's records,
    verification against them, the records of the target rows kept, and the
    draft distilled from these at each first rejection."""
    import torch
    B, K, V, k, T = 9, 4, 12007, 64, 1.0
    t = as_dtype(rows("normal", B * (K + 1), V, 300), dtype).reshape(B, K + 1, V)
    d = as_dtype(topk_ref.values(t[:, :K]).astype(np.float32) + rows("normal", B * K, V, 301).reshape(B, K, V) / 4,
                 dtype)
    ud, ua, ur = uniforms((K, B), 302), uniforms((B, K), 303), uniforms(B, 304)
    dt, dd = to_device(t), to_device(d)
    ids = torch.empty(B, K, k, dtype=torch.int32, device="cuda")
    top = torch.empty(B, K, k, dtype=dd.dtype, device="cuda")
    y = torch.empty(B, K, dtype=torch.int32, device="cuda")
    for i in range(K):  # the draft's autoregressive steps
        ids[:, i], top[:, i], _, y[:, i] = osd.osd_topk(dd[:, i, :], k, T, to_device(ud[i]), rest=False)
    acc, toks, rmask = osd.osd_verify_topk(dt, ids, top, y, to_device(ua), to_device(ur), T)
    ti, tt, tr, _ = osd.osd_topk(dt.view(-1, V), k, T)
    loss, rl, g = osd.osd_distill_topk_loss_grad(ti.view(B, K + 1, k), tt.view(B, K + 1, k), tr.view(B, K + 1), dd,
                                                 "fkl", 0.5, T, mask=rmask)
    x = dict(t=t, ids=host(ids), top=host(top), y=host(y), ua=ua, ur=ur)
    rec = topk_ref.topk(d.transpose(1, 0, 2).reshape(K * B, V), k, T, ud.reshape(-1))
    assert np.array_equal(x["y"], rec["tokens"].reshape(K, B).T)
    check((acc, toks, rmask), x, T, None, "step")
    from tests.test_distill_topk_gpu import check as check_distill
    from tests.test_distill_topk_gpu import record
    fi, ft, fr = record(t[:, :K].reshape(B * K, V), k, T)
    check_distill((loss, rl, g), fi, ft, fr, d.reshape(B * K, V), "fkl", 0.5, T, host(rmask), "step")


def flat_rows(V, gap, dtype, seed, kind):
    """[8, V] rows whose terms round alike: one head token far above equal others
    (first, last or in the middle), in one stretch of the row or all over it; or
    eight logits over and over, other ones in the second half."""
    g = np.random.default_rng(seed)
    x = np.full((8, V), -gap, np.float32)
    for n in range(8):
        if kind == "pattern":
            half = V // 2 // 8 * 8
            for lo, hi in ((0, half), (half, V)):
                x[n, lo:hi] = np.resize(-gap * g.random(8), hi - lo)
        elif kind == "stretch":  # one stretch of at most 2048 tokens
            x[n] = -np.inf
            lo = int(g.integers(0, max(1, V // 2048))) * 2048
            x[n, lo:lo + 2047] = -gap
        if kind != "pattern":
            x[n, [0, V - 1, int(g.integers(V))][n % 3]] = 0.0
    return as_dtype(x, dtype)


FLAT = [(2048, 6.84375), (1024, 6.4375), (2047, 7.625), (4099, 8.3125), (32003, 10.375), (65536, 11.0625)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1.0, 0.875, 0.6])
@pytest.mark.parametrize("kind", ["head", "stretch", "pattern"])
@pytest.mark.parametrize("V,gap", FLAT)
def test_draws_next_to_edges_of_flat_rows(osd, V, gap, kind, T, dtype):
    """Uniforms next to the edges of tokens' intervals, where the errors of equal
    terms add up: the bonus token, and the correction after a proposal that the
    target has as good as no mass for."""
    T = float(np.float32(T))
    t = flat_rows(V, gap if dtype == "bf16" else np.float32(gap * 1.0437), dtype, V, kind)
    z = topk_ref.values(t)
    g = np.random.default_rng(V + 1)
    n = 96 if V < 5000 else 32
    which = g.integers(0, 8, n)
    ids = np.zeros((n, 1, 1), np.int32)
    ur = np.zeros((2, n), np.float32)
    for b in range(n):
        p = topk_ref.softmax(z[which[b]] / T)
        some = np.nonzero(p > 0)[0]
        y = ids[b, 0, 0] = some[g.integers(len(some))]
        for corrected in range(2):
            if corrected:  # the proposal's draft mass is 1
                p[y] = 0.0
            edge = np.float32(np.cumsum(p)[some[g.integers(len(some))]] / p.sum()) + np.float32(
                int(g.integers(-6, 7)) * 2.0 ** -24)
            ur[corrected, b] = np.clip(edge, np.float32(0), np.float32(1 - 2.0 ** -24))
    pair = np.stack([t[which], t[which]], 1)
    x = dict(t=pair, ids=ids, top=np.zeros((n, 1, 1), t.dtype), y=ids[:, :, 0], ua=np.zeros((n, 1), np.float32),
             ur=ur[0])
    left = check(call(osd, x, T), x, T, None, f"bonus {kind} V={V} T={T} {dtype}")
    x["ua"][:] = np.float32(1 - 2.0 ** -24)
    x["ur"] = ur[1]
    left += check(call(osd, x, T), x, T, None, f"correction {kind} V={V} T={T} {dtype}")
    # (Where tokens have 1e-8 of the mass, one point in five is within 1e-9 of an edge on either side.)
    assert left <= n  # of 2 n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1.0, 0.875, 0.75, 0.6])
@pytest.mark.parametrize("V,gap", FLAT)
def test_acceptance_next_to_the_ratio(osd, V, gap, T, dtype):
    """Uniforms next to p(y) / q(y), the head proposed from a record of its own."""
    T = float(np.float32(T))
    t = flat_rows(V, gap if dtype == "bf16" else np.float32(gap * 1.0437), dtype, V, "head")
    n = 64
    which = np.arange(n) % 8
    p = np.array([topk_ref.softmax(r / T).max() for r in topk_ref.values(t)])
    y = np.array([int(np.argmax(r)) for r in topk_ref.values(t)], np.int32)[which]
    ua = p[which].astype(np.float32)
    for b in range(n):
        for _ in range(b // 8):
            ua[b] = np.nextafter(ua[b], np.float32(0 if b % 2 else 1), dtype=np.float32)
    x = dict(t=np.stack([t[which], t[which]], 1), ids=y.reshape(n, 1, 1), top=np.zeros((n, 1, 1), t.dtype),
             y=y.reshape(n, 1), ua=ua.reshape(n, 1), ur=uniforms(n, 5))
    check(call(osd, x, T), x, T, None, f"V={V} T={T} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e-38, 1e-30, 1e-4, 300.0, 1e30, 1e37, 3.0e38])
@pytest.mark.parametrize("V", [5, 1001, 33000])
def test_extreme_temperatures_and_masks(osd, V, T, dtype):
    """Temperatures at which log2(e) / T or its parts leave the range of floats, on
    rows with masked tokens (-inf, the lowest finite value), at the row's ragged end
    too; small and large logits."""
    T = float(np.float32(T))
    B, K, k = 12, 2, 4
    g = np.random.default_rng(V)
    t = rows("normal", B * (K + 1), V, V).reshape(B, K + 1, V)
    t[g.random(t.shape) < 0.3] = -np.inf
    t[2:4, :, : V // 2] = lowest(dtype)
    t[4:6, :, V // 2 :] = -np.inf
    t[6:8] *= np.float32(1e-20)
    t[8:10] *= np.float32(1e20)
    t[:, :, V // 3] = 0.25
    d = as_dtype(t[:, :K].reshape(B * K, V).copy(), dtype)
    t = as_dtype(t, dtype)
    rec = topk_ref.topk(d, k, T, uniforms(B * K, 1))
    top = np.where(rec["ids"] < 0, as_dtype(np.full((1, 1), -np.inf, np.float32), dtype),
                   np.take_along_axis(d, np.maximum(rec["ids"], 0).astype(np.int64), 1))
    x = dict(t=t, ids=rec["ids"].reshape(B, K, k), top=top.reshape(B, K, k), y=rec["tokens"].reshape(B, K),
             ua=uniforms((B, K), 2), ur=uniforms(B, 3))
    with np.errstate(over="ignore"):
        check(call(osd, x, T), x, T, None, f"V={V} T={T} {dtype}")


@pytest.mark.parametrize("T", [1.0, 0.875, 0.75, 0.6])
def test_residual_of_one_token_with_little_mass(osd, T):
    """A draft that is the target but for one token, which it lacks: at u next to 1
    a proposal is rejected, and that token is the correction however little mass it
    has (fp32 masses leave less than their rounding, or nothing).  The record: one
    logit far above 255 equal ones, or any."""
    V, k, n = 1000, 256, 160
    T = float(np.float32(T))
    g = np.random.default_rng(3)
    t = np.full((n, 2, V), -np.inf, np.float32)
    ids = np.stack([np.sort(g.choice(V, k, replace=False)) for _ in range(n)]).astype(np.int32)
    top = g.normal(0, 2, (n, k)).astype(np.float32)
    left = np.zeros(n, np.int64)
    for b in range(n):
        if b % 4:
            top[b] = -T * (np.log(k - 1) + g.random())
            top[b, g.integers(k)] = 0.0
        left[b] = g.choice(np.setdiff1d(np.arange(V), ids[b]))
        t[b, :, ids[b]] = top[b][:, None]
        mass = np.exp(top[b].astype(np.float64) / T).sum()
        t[b, :, left[b]] = T * np.log(mass * np.geomspace(7e-8, 1e-6, n)[b])
    x = dict(t=t, ids=ids.reshape(n, 1, k), top=top.reshape(n, 1, k), y=ids[np.arange(n), top.argmax(1)].reshape(n, 1),
             ua=np.full((n, 1), 1 - 2.0 ** -24, np.float32), ur=uniforms(n, 4))
    acc, toks, rmask = (host(o) for o in call(osd, x, T))
    wa, wt, wm, margin = topk_ref.verify(x["t"], x["ids"], x["top"], x["y"], x["ua"], x["ur"], T)
    sure = margin > 1e-10  # (the fp64 exponentials are within 1e-12)
    assert sure.sum() > n // 2 and (wa[sure] == 0).all() and (wt[sure, 0] == left[sure]).all()
    bad = sure & ((acc != wa) | (toks[:, 0] != wt[:, 0]))
    assert not bad.any(), f"{bad.sum()}: {acc[bad]} {toks[bad, 0]} for {wt[bad, 0]}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1e6, 1e9, 1e20])
def test_large_logits_at_large_temperatures(osd, T, dtype):
    """Logits whose products with their exponentials leave fp32 although the scaled
    logits are ordinary ones (60 to 99 bits), with and without masked tokens."""
    T = float(np.float32(T))
    B, K, V, k = 8, 2, 5001, 8
    g = np.random.default_rng(9)
    t = (g.uniform(-99, 99, (B, K + 1, V)) * T * np.log(2)).astype(np.float32)
    t[:4][g.random((4, K + 1, V)) < 0.3] = -np.inf
    t[2:6, :, 3] = np.float32(98.5 * T * np.log(2))
    d = as_dtype(t[:, :K].reshape(B * K, V).copy(), dtype)
    t = as_dtype(t, dtype)
    rec = topk_ref.topk(d, k, T, uniforms(B * K, 1))
    top = np.take_along_axis(d, rec["ids"].astype(np.int64), 1)
    x = dict(t=t, ids=rec["ids"].reshape(B, K, k), top=top.reshape(B, K, k), y=rec["tokens"].reshape(B, K),
             ua=uniforms((B, K), 2), ur=uniforms(B, 3))
    check(call(osd, x, T), x, T, None, f"T={T} {dtype}")
    x["ua"][:] = 0.0
    check(call(osd, x, T), x, T, None, f"bonus T={T} {dtype}")


@pytest.mark.parametrize("kind", ["head", "pattern"])
@pytest.mark.parametrize("V,gap", [(100003, 11.5), (131072, 11.75)])
def test_draws_next_to_edges_of_the_longest_bf16_rows(osd, V, gap, kind):
    test_draws_next_to_edges_of_flat_rows(osd, V, gap, kind, 1.0, "bf16")
    if kind == "head":
        test_acceptance_next_to_the_ratio(osd, V, gap, 1.0, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [2, 5, 16])
def test_every_position_next_to_its_ratio(osd, K, dtype):
    """Uniforms next to p(y) / q(y) at all positions: one after another is decided
    in fp64, the first that fails ends it; ragged lengths."""
    V, gap, T, B = 2048, 6.84375, 1.0, 40
    t = flat_rows(V, gap, dtype, V, "head")
    z = topk_ref.values(t)
    which = (np.arange(B * K).reshape(B, K) + np.arange(B)[:, None]) % 8
    p = np.array([topk_ref.softmax(r / T).max() for r in z])
    y = np.array([int(np.argmax(r)) for r in z], np.int32)[which]
    ua = p[which].astype(np.float32)
    for b in range(B):
        for i in range(K):  # accepted up to position b % (K + 1)
            for _ in range(1 + (b + i) % 3):
                ua[b, i] = np.nextafter(ua[b, i], np.float32(0 if i < b % (K + 1) else 1), dtype=np.float32)
    rows_t = np.concatenate([t[which], t[which[:, :1]]], 1)
    x = dict(t=rows_t, ids=y.reshape(B, K, 1), top=np.zeros((B, K, 1), t.dtype), y=y, ua=ua, ur=uniforms(B, 5))
    check(call(osd, x, T), x, T, None, f"K={K} {dtype}")
    dl = (np.arange(B) % K + 1).astype(np.int32)
    check(call(osd, x, T, dl), x, T, dl, f"ragged K={K} {dtype}")
    acc = host(call(osd, x, T)[0])
    assert set(acc.tolist()) == set(range(K + 1))


def test_masked_rows_and_other_sizes_on_one_workspace(osd):
    """Calls of several K, V and types in turn through the binding's workspace: what
    one leaves there does not reach the next."""
    import torch
    calls = []
    for n, (B, K, V, k, dtype, kind) in enumerate([(6, 16, 3001, 40, "bf16", "masked"), (3, 1, 70001, 7, "bf16", "normal"),
                                                   (40, 5, 2048, 256, "f32", "equal"), (2, 3, 5, 2, "bf16", "normal"),
                                                   (9, 2, 40003, 33, "f32", "masked_lowest")]):
        x = inputs(B, K, V, k, dtype, 1.0, 400 + n, kind=kind)
        calls.append((x, call(osd, x, 1.0)))
        check(calls[-1][1], x, 1.0, None, f"{kind} V={V}")
    for x, first in calls[::-1] + calls:
        assert all(torch.equal(a, b) for a, b in zip(call(osd, x, 1.0), first))
