"""osd_distill_topk_loss_grad against the 64-bit reference.

Tolerances: the logarithm of the others' mass is within LOG_SUM (see
_topk_helpers), and each log ratio and D with it; a gradient is q_j times a
factor made of these, q_j to 2^-16 (the exponent's rounding over 2^-64) and one
rounding to the type (half a step: 2^-8 relative for bf16, 2^-24 for fp32).  RKL
and JSD multiply LOG_SUM by log ratios, at most 40 here, weighted by q.
"""
import numpy as np
import pytest

from oracle import topk_ref
from tests._helpers import to_device
from tests._topk_helpers import LOG_SUM, as_dtype, lowest, rows
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


def record(t, k, tau):
    rec = topk_ref.topk(t, k, tau)
    top = np.take_along_axis(t, np.maximum(rec["ids"], 0).astype(np.int64), 1)
    ninf = np.uint16(0xFF80) if t.dtype == np.uint16 else np.float32(-np.inf)
    return rec["ids"], np.where(rec["ids"] < 0, ninf, top), rec["rest"].astype(np.float32)


def check(got, ids, top, rest, s, kind, beta, tau, mask, label):
    loss, rl, g = (host(t) for t in got)
    N, V = s.shape
    wl, wr, wg = topk_ref.distill(ids, top, rest, s, kind, beta, tau, mask)
    on = np.ones(N, bool) if mask is None else mask.reshape(-1) != 0
    ok = np.isfinite(wr)
    if rl is not None:
        rl = rl.reshape(-1)
        assert np.array_equal(np.isnan(rl), np.isnan(wr)), f"{label}: NaN rows"
        assert np.array_equal(rl[np.isinf(wr)], wr[np.isinf(wr)]), f"{label}: infinite rows"
        err = np.abs(rl[ok] - wr[ok])
        lim = 4 * LOG_SUM + 1e-5 * np.abs(wr[ok])
        assert (err <= lim).all(), f"{label}: row loss off by {err.max()} of {wr[ok][err.argmax()]}"
        assert (rl[~on] == 0).all()
    if ok.all():
        assert np.allclose(loss, wl, rtol=1e-5, atol=4 * LOG_SUM * max(1, int(on.sum()))), f"{label}: loss {loss} {wl}"
    elif np.isnan(wr).any():
        assert np.isnan(loss).all()
    if g is not None:
        g = topk_ref.values(g.reshape(N, V))
        assert np.array_equal(np.isnan(g[~ok]), np.isnan(wg[~ok])), f"{label}: NaN gradients"
        step = 2.0 ** -8 if s.dtype == np.uint16 else 2.0 ** -24
        tiny = 2.0 ** -133 if s.dtype == np.uint16 else 2.0 ** -149
        lim = (step + 2.0 ** -15) * np.abs(wg[ok]) + 40 * LOG_SUM * qof(s[ok], tau) / tau + tiny
        err = np.abs(g[ok] - wg[ok])
        bad = err > lim
        assert not bad.any(), f"{label}: {bad.sum()} gradients, {g[ok][bad][:3]} for {wg[ok][bad][:3]}"
        assert (g[~on] == 0).all(), f"{label}: masked rows"


def qof(s, tau):
    x = topk_ref.values(s) / tau
    with np.errstate(invalid="ignore"):
        e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def call(osd, ids, top, rest, s, B, K, kind, beta, tau, mask=None, **kw):
    V, k = s.shape[1], ids.shape[1]
    return osd.osd_distill_topk_loss_grad(
        to_device(ids.reshape(B, -1, k)), to_device(top.reshape(B, -1, k)),
        None if rest is None else to_device(rest.reshape(B, -1)), to_device(s.reshape(B, K, V)), kind, beta, tau,
        mask=None if mask is None else to_device(mask.reshape(B, K)), **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("V,k", [(1, 1), (2, 1), (7, 7), (9, 4), (100, 64), (1001, 65), (2048, 256), (4099, 1),
                                 (8192, 100), (16384, 64), (20011, 33), (32000, 64), (32771, 255)])
def test_shapes(osd, V, k, kind, dtype):
    B, K, tau, beta = 3, 2, 0.75, 0.25
    t = as_dtype(rows("normal", B * K, V, V), dtype)
    s = as_dtype(topk_ref.values(t).astype(np.float32) + rows("normal", B * K, V, V + 1) / 3, dtype)
    ids, top, rest = record(t, k, tau)
    for r in ((rest, None) if kind != "rkl" and k < V else (rest,)):
        got = call(osd, ids, top, r, s, B, K, kind, beta, tau)
        check(got, ids, top, r, s, kind, beta, tau, None, f"V={V} k={k} {kind} {dtype} rest={r is not None}")


@pytest.mark.parametrize("V,k,dtype,kind", [(65536, 100, "f32", "rkl"), (50257, 20, "f32", "jsd"),
                                            (131072, 256, "bf16", "fkl"), (128256, 64, "bf16", "jsd"),
                                            (100003, 17, "bf16", "rkl")])
def test_long_rows(osd, V, k, dtype, kind):
    B, K, tau, beta = 1, 3, 1.0, 0.5
    t = as_dtype(rows("normal", B * K, V, V), dtype)
    s = as_dtype(topk_ref.values(t).astype(np.float32) + rows("normal", B * K, V, V + 1) / 3, dtype)
    ids, top, rest = record(t, k, tau)
    got = call(osd, ids, top, rest, s, B, K, kind, beta, tau)
    check(got, ids, top, rest, s, kind, beta, tau, None, f"V={V} k={k} {kind} {dtype}")


@pytest.mark.parametrize("V,k,dtype,B", [(12289, 33, "bf16", 200), (30011, 64, "bf16", 200), (50257, 64, "bf16", 200),
                                         (128256, 256, "bf16", 150), (5003, 200, "f32", 300), (9001, 64, "f32", 300),
                                         (32003, 20, "f32", 200), (65536, 100, "f32", 150)])
def test_many_rows_each_as_if_alone(osd, V, k, dtype, B):
    """Five rows over and over, so that there are many: each repeat has the bits
    of the first, and those are right; without the gradient too."""
    import torch
    n, tau = 5, 1.0
    t = as_dtype(rows("normal", n, V, V + 2), dtype)
    s = as_dtype(rows("normal", n, V, V + 3), dtype)
    ids, top, rest = record(t, k, tau)
    d = [to_device(a) for a in (ids, top, rest, s)]
    for kind in ("fkl", "rkl", "jsd"):
        ids_d, top_d, rest_d, s_d = (x.repeat((B // n,) + (1,) * (x.dim() - 1)) for x in d)
        args = (ids_d.view(B, 1, k), top_d.view(B, 1, k), rest_d.view(B, 1), s_d.view(B, 1, V), kind, 0.5, tau)
        loss, rl, g = osd.osd_distill_topk_loss_grad(*args)
        assert torch.equal(rl.view(-1, n), rl[:n].view(1, n).expand(B // n, n))
        assert torch.equal(g.view(-1, n, V), g[:n].view(1, n, V).expand(B // n, n, V))
        alone = loss.clone()
        alone[1] = alone[1] * n / B
        check((alone, rl[:n], g[:n]), ids, top, rest, s, kind, 0.5, tau, None, f"V={V} k={k} {kind} {dtype} B={B}")
        loss, rl, g = osd.osd_distill_topk_loss_grad(*args, grad=False)
        alone = loss.clone()
        alone[1] = alone[1] * n / B
        assert torch.equal(rl.view(-1, n), rl[:n].view(1, n).expand(B // n, n))
        check((alone, rl[:n], None), ids, top, rest, s, kind, 0.5, tau, None, f"no grad V={V} k={k} {kind} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("B", [1, 37, 700])
def test_masks_and_row_counts(osd, B, kind, dtype):
    K, V, k, tau, beta = 3, 1001, 20, 1.0, 0.5
    t = as_dtype(rows("normal", B * K, V, 3), dtype)
    s = as_dtype(rows("normal", B * K, V, 4), dtype)
    ids, top, rest = record(t, k, tau)
    g = np.random.default_rng(5)
    for mask in ((g.random((B, K)) < 0.4).astype(np.uint8), np.zeros((B, K), np.uint8), None):
        got = call(osd, ids, top, rest, s, B, K, kind, beta, tau, mask)
        check(got, ids, top, rest, s, kind, beta, tau, mask, f"B={B} {kind} {dtype}")
        again = call(osd, ids, top, rest, s, B, K, kind, beta, tau, mask)
        import torch
        assert all(torch.equal(a, b) for a, b in zip(got, again)), "equal calls, unequal bits"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("student", ["ties", "equal", "lowest", "masked", "masked_lowest", "peak", "bad"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("V", [3001, 12007])
def test_student_kinds(osd, V, student, kind, dtype):
    """Masked vocabularies (-inf, the type's lowest), rows of equal logits,
    rows without a softmax."""
    B, K, k, tau, beta = 5, 1, 33, 1.0, 0.5
    t = as_dtype(rows("normal", B, V, 6), dtype)
    s = as_dtype(rows(student, B, V, 7, dtype), dtype)
    ids, top, rest = record(t, k, tau)
    if student == "masked_lowest":  # differences of 1e38: only their sign is compared
        got = call(osd, ids, top, rest, s, B, K, kind, beta, tau)
        _, wr, _ = topk_ref.distill(ids, top, rest, s, kind, beta, tau)
        rl = host(got[1]).reshape(-1)
        assert np.allclose(rl, wr, rtol=1e-4, atol=1e-4)
        return
    got = call(osd, ids, top, rest, s, B, K, kind, beta, tau)
    check(got, ids, top, rest, s, kind, beta, tau, None, f"{student} {kind} {dtype}")


@pytest.mark.parametrize("V", [2003, 12007])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
def test_teacher_kinds_and_bad_records(osd, kind, V):
    """Rows whose teacher is masked to fewer tokens than slots, uniform, or has
    no record; records with an id twice, out of range, NaN, +inf, an empty first
    slot."""
    k, tau, beta = 40, 1.0, 0.5
    for tk in ("masked", "lowest", "equal", "bad"):
        t, s = as_dtype(rows(tk, 6, V, 8, "f32"), "f32"), as_dtype(rows("normal", 6, V, 9), "f32")
        if tk == "masked":
            keep = np.random.default_rng(1).choice(V, k // 2, replace=False)
            t[:] = -np.inf
            t[:, keep] = rows("normal", 6, k // 2, 10)
            t[1] = -np.inf
        ids, top, rest = record(t, k, tau)
        got = call(osd, ids, top, rest, s, 6, 1, kind, beta, tau)
        check(got, ids, top, rest, s, kind, beta, tau, None, f"teacher {tk} {kind}")
    t, s = as_dtype(rows("normal", 9, V, 11), "bf16"), as_dtype(rows("normal", 9, V, 12), "bf16")
    ids, top, rest = record(t, k, tau)
    ids, top, rest = ids.copy(), top.copy(), rest.copy()
    ids[0, 7] = ids[0, 39]
    ids[1, 3] = V
    ids[2, 3] = -2
    ids[3, 3] = 0x7FFFFFFF
    top[4, 5] = 0x7FC0
    top[5, 0] = 0x7F80
    ids[6, 0], top[6, 0] = -1, 0xFF80
    rest[7] = np.nan
    got = call(osd, ids, top, rest, s, 9, 1, kind, beta, tau)
    check(got, ids, top, rest, s, kind, beta, tau, None, f"bad records {kind}")
    mask = np.ones((9, 1), np.uint8)
    mask[:8] = 0
    got = call(osd, ids, top, rest, s, 9, 1, kind, beta, tau, mask)
    check(got, ids, top, rest, s, kind, beta, tau, mask, f"bad records masked {kind}")
    assert np.isfinite(host(got[0])).all()


@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_jsd_endpoints_exactly_zero(osd, beta):
    t, s = as_dtype(rows("normal", 4, 999, 13), "bf16"), as_dtype(rows("masked", 4, 999, 14), "bf16")
    ids, top, rest = record(t, 20, 1.0)
    for r in (rest, None):
        loss, rl, g = call(osd, ids, top, r, s, 4, 1, "jsd", beta, 1.0)
        assert (loss == 0).all() and (rl == 0).all() and (g == 0).all()


def test_whole_row_record_matches_osd_distill(osd):
    """k = V: the whole rows' divergence."""
    B, K, V = 4, 2, 200
    t, s = as_dtype(rows("normal", B * K, V, 15), "f32"), as_dtype(rows("normal", B * K, V, 16), "f32")
    ids, top, rest = record(t, V, 1.0)
    for kind in ("fkl", "rkl", "jsd"):
        a = call(osd, ids, top, rest, s, B, K, kind, 0.5, 1.0)
        b = osd.osd_distill_loss_grad(to_device(t.reshape(B, K, V)), to_device(s.reshape(B, K, V)), kind, 0.5, 1.0)
        # both within 1e-5 of the exact value
        assert np.allclose(host(a[1]), host(b[1]), rtol=2e-5, atol=1e-6)
        assert np.allclose(host(a[2]), host(b[2]), rtol=2e-5, atol=4e-6)


@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
def test_gradient_by_differences(osd, kind):
    """(D(s + h) - D(s - h)) / 2h of the kernel's own row losses, in tokens of
    the record and outside it.  With h = 2^-4 the loss's error (4 LOG_SUM +
    1e-5 D) makes (4e-6 + 1e-5 D) / h of the quotient, the third derivative
    (at most 8 / tau^3 here) h^2 / 6 times that."""
    V, k, tau, h = 50, 8, 1.0, 2.0 ** -4
    t, s = rows("normal", 1, V, 17) / 2, rows("normal", 1, V, 18) / 2
    ids, top, rest = record(t, k, tau)
    g = host(call(osd, ids, top, rest, s, 1, 1, kind, 0.5, tau)[2]).reshape(-1)
    picks = [int(ids[0, 0]), int(ids[0, 7])] + [j for j in range(V) if j not in ids[0]][:4]
    both = np.repeat(s, 2 * len(picks), 0)
    for i, j in enumerate(picks):
        both[2 * i, j] += np.float32(h)
        both[2 * i + 1, j] -= np.float32(h)
    n = len(both)
    rl = host(call(osd, np.repeat(ids, n, 0), np.repeat(top, n, 0), np.repeat(rest, n), both, n, 1, kind, 0.5,
                   tau)[1]).reshape(-1).astype(np.float64)
    for i, j in enumerate(picks):
        step = float(both[2 * i, j]) - float(both[2 * i + 1, j])
        lim = (4.8e-6 + 1e-5 * abs(rl).max()) / h + 8 * h * h / 6
        assert abs((rl[2 * i] - rl[2 * i + 1]) / step - g[j]) < lim


def test_optional_outputs_strides_and_in_place(osd):
    """K of K+1 records per sequence, a student with a batch stride, outputs
    left out, the gradient in the student rows' own place."""
    import torch
    B, K, V, k = 5, 3, 2001, 16
    for dtype in ("bf16", "f32"):
        t = as_dtype(rows("normal", B * (K + 1), V, 19), dtype)
        s4 = as_dtype(rows("normal", B * (K + 1), V, 20), dtype).reshape(B, K + 1, V)
        s = np.ascontiguousarray(s4[:, :K]).reshape(B * K, V)
        ids, top, rest = record(t, k, 1.0)
        first = lambda a: np.ascontiguousarray(a.reshape(B, K + 1, -1)[:, :K]).reshape(B * K, -1)
        fi, ft, fr = first(ids), first(top), first(rest).reshape(-1)
        dev = [to_device(a) for a in (ids.reshape(B, K + 1, k), top.reshape(B, K + 1, k), rest.reshape(B, K + 1))]
        ds = to_device(s4)[:, :K]
        got = osd.osd_distill_topk_loss_grad(*dev, ds, "jsd", 0.5, 1.0)
        check(got, fi, ft, fr, s, "jsd", 0.5, 1.0, None, f"strides {dtype}")
        got2 = osd.osd_distill_topk_loss_grad(*dev, ds, "jsd", 0.5, 1.0, grad=False, row_loss=False)
        assert got2[1] is None and got2[2] is None and torch.equal(got2[0], got[0])
        own = ds.contiguous()
        osd.osd_distill_topk_loss_grad(*dev, own, "jsd", 0.5, 1.0, out=(torch.empty(2, device="cuda"), None, own))
        assert torch.equal(own, got[2])
        room = torch.cat([ds.reshape(-1), ds.reshape(-1)[:V]])  # a gradient one row further on
        with pytest.raises(osd.OsdError):
            osd.osd_distill_topk_loss_grad(*dev, room[:B * K * V].view(B, K, V), "jsd", 0.5, 1.0,
                                           out=(torch.empty(2, device="cuda"), None, room[V:].view(B, K, V)))


def test_long_rows_in_place(osd):
    import torch
    B, K, V, k = 2, 1, 100003, 64
    t, s = as_dtype(rows("normal", 2, V, 21), "bf16"), as_dtype(rows("normal", 2, V, 22), "bf16")
    ids, top, rest = record(t, k, 1.0)
    a = call(osd, ids, top, rest, s, B, K, "fkl", 0.5, 1.0)
    check(a, ids, top, rest, s, "fkl", 0.5, 1.0, None, "long")
    own = to_device(s.reshape(B, K, V))
    b = osd.osd_distill_topk_loss_grad(to_device(ids.reshape(B, K, k)), to_device(top.reshape(B, K, k)),
                                       to_device(rest.reshape(B, K)), own, "fkl", 0.5, 1.0,
                                       out=(torch.empty(2, device="cuda"), torch.empty(B, K, device="cuda"), own))
    check(b, ids, top, rest, s, "fkl", 0.5, 1.0, None, "long in place")


def test_guard_bands(osd):
    import ctypes
    import torch
    from paper_2310_07177_amd import binding
    for B, K, V, k, dtype in [(2, 2, 7, 3, "bf16"), (3, 1, 1001, 20, "f32"), (2, 3, 32003, 64, "bf16"),
                              (1, 2, 70001, 64, "bf16")]:
        n = B * K
        t, s = as_dtype(rows("normal", n, V, 23), dtype), as_dtype(rows("normal", n, V, 24), dtype)
        ids, top, rest = record(t, k, 1.0)
        d = [to_device(a) for a in (ids, top, rest, s)]
        es = d[3].element_size()
        sizes = [8, n * 4, n * V * es]
        bufs = [torch.full((z + 8192,), 0x5A, dtype=torch.uint8, device="cuda") for z in sizes]
        size = osd.lib().osd_distill_topk_workspace_bytes(B, K)
        ws = torch.zeros(size + 8192, dtype=torch.uint8, device="cuda")
        ws[:4096] = ws[4096 + size:] = 0x5A
        p = lambda x, o=0: ctypes.c_void_p(x.data_ptr() + o)
        st = osd.lib().osd_distill_topk_loss_grad(
            p(d[0]), p(d[1]), p(d[2]), K, k, p(d[3]), K * V, binding.OSD_BF16 if es == 2 else binding.OSD_F32, B, K,
            V, None, 2, 0.5, 1.0, p(bufs[0], 4096), p(bufs[1], 4096), p(bufs[2], 4096), p(ws, 4096), size, None)
        assert st == 0
        torch.cuda.synchronize()
        for b, z in zip(bufs + [ws], sizes + [size]):
            assert (b[:4096] == 0x5A).all() and (b[4096 + z:] == 0x5A).all()


def test_one_workspace_at_many_sizes(osd):
    """What a call leaves in the workspace does not reach later calls of other
    sizes, rows split over workgroups or not."""
    import ctypes
    import torch
    from paper_2310_07177_amd import binding
    shapes = [(4, 3, 32003, 64, "bf16"), (1, 1, 70001, 8, "bf16"), (3, 1, 1001, 20, "f32"), (31, 20, 2500, 256, "f32"),
              (2, 3, 50257, 256, "f32"), (1, 2, 300, 300 - 44, "bf16"), (40, 10, 9001, 33, "bf16")]
    calls = []
    for B, K, V, k, dtype in shapes:
        n = B * K
        t, s = as_dtype(rows("normal", n, V, 51), dtype), as_dtype(rows("normal", n, V, 52), dtype)
        ids, top, rest = record(t, k, 1.0)
        d = [to_device(a) for a in (ids, top, rest, s)]
        out = [torch.empty(z, dtype=torch.uint8, device="cuda") for z in (8, n * 4, n * V * d[3].element_size())]
        calls.append((B, K, V, k, d, out))
    size = max(osd.lib().osd_distill_topk_workspace_bytes(B, K) for B, K, *_ in shapes)

    def run(call, ws):
        B, K, V, k, d, out = call
        p = lambda x: ctypes.c_void_p(x.data_ptr())
        st = osd.lib().osd_distill_topk_loss_grad(
            p(d[0]), p(d[1]), p(d[2]), K, k, p(d[3]), K * V,
            binding.OSD_BF16 if d[3].element_size() == 2 else binding.OSD_F32, B, K, V, None, 2, 0.5, 1.0, p(out[0]),
            p(out[1]), p(out[2]), p(ws), ws.numel(), None)
        assert st == 0
        torch.cuda.synchronize()
        return [o.clone() for o in out]

    want = [run(c, torch.zeros(size, dtype=torch.uint8, device="cuda")) for c in calls]
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for c, w in zip(calls, want):
            for g, x in zip(run(c, ws), w):
                assert (g == x).all(), c[:4]


@pytest.mark.parametrize("V", [5003, 20011])
def test_graph(osd, V):
    import torch
    B, K, k = 9, 4, 32
    data = []
    for i in range(3):
        t, s = as_dtype(rows("normal", B * K, V, 30 + i), "bf16"), as_dtype(rows("normal", B * K, V, 40 + i), "bf16")
        ids, top, rest = record(t, k, 1.0)
        data.append([to_device(a) for a in (ids.reshape(B, K, k), top.reshape(B, K, k), rest.reshape(B, K),
                                            s.reshape(B, K, V))])
    held = [d.clone() for d in data[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        osd.osd_distill_topk_loss_grad(*held, "rkl", 0.5, 1.0)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = osd.osd_distill_topk_loss_grad(*held, "rkl", 0.5, 1.0)
    for i in (1, 2, 0, 1):
        for h, d in zip(held, data[i]):
            h.copy_(d)
        eager = osd.osd_distill_topk_loss_grad(*held, "rkl", 0.5, 1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("B,V", [(3, 3001), (3, 12007), (150, 12007)])
def test_others_far_below_the_record(osd, B, V, kind, dtype):
    """A student whose mass outside the record is far below what 32 bits hold:
    the others still share the teacher's rest."""
    k, tau = 33, 1.0
    t = as_dtype(rows("normal", 3, V, 70), dtype)
    ids, top, rest = record(t, k, tau)
    for gap in (60.0, 88.0, 95.0, 200.0, 600.0):
        s = rows("normal", 3, V, 71) - np.float32(gap)
        for n in range(3):
            s[n, ids[n]] += np.float32(gap)
        s = as_dtype(s, dtype)
        ti, tt, tr, ts = (np.concatenate([a] * (B // 3)) for a in (ids, top, rest, s))
        loss, rl, g = call(osd, ti, tt, tr, ts, B, 1, kind, 0.5, tau)
        loss = loss.clone()
        loss[1] = loss[1] * 3 / B
        check((loss, rl[:3], g[:3]), ids, top, rest, s, kind, 0.5, tau, None, f"gap {gap} {kind} {dtype}")


def test_lowest_of_the_type(osd):
    """A teacher and a student that are the type's lowest value everywhere are
    uniform: D = 0."""
    V, k = 1000, 10
    for dtype in ("bf16", "f32"):
        x = as_dtype(np.full((2, V), lowest(dtype), np.float32), dtype)
        ids, top, rest, _ = osd.osd_topk(to_device(x), k, 1.0)
        assert np.allclose(host(rest), np.log(V - k), atol=1e-5)
        loss, rl, g = osd.osd_distill_topk_loss_grad(ids.view(2, 1, k), top.view(2, 1, k), rest.view(2, 1),
                                                     to_device(x.reshape(2, 1, V)), "fkl")
        assert np.abs(host(rl)).max() < 4 * LOG_SUM


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("B,V", [(3, 3001), (3, 12007), (150, 12007)])
def test_others_below_64_bits(osd, B, V, kind, dtype):
    """The same where the others' mass leaves fp64's range too (a student masked
    with -1e4): the loss is finite, and the gradient that loss's own: a row's
    gradients add up to 0, those outside the record in FKL to Q - P, Q = 0.

    Sums: each gradient is off by half a step of the type and 2^-15 of itself, and
    all by 40 LOG_SUM q (see above), which adds up to these of the sum of their
    magnitudes and 40 LOG_SUM."""
    k, tau = 33, 1.0
    t = as_dtype(rows("normal", 3, V, 80), dtype)
    ids, top, rest = record(t, k, tau)
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for gap in (700.0, 740.0, 760.0, 900.0, 1.0e4):
        s = rows("normal", 3, V, 81) - np.float32(gap)
        for n in range(3):
            s[n, ids[n]] += np.float32(gap)
        s = as_dtype(s, dtype)
        ti, tt, tr, ts = (np.concatenate([a] * (B // 3)) for a in (ids, top, rest, s))
        loss, rl, g = call(osd, ti, tt, tr, ts, B, 1, kind, 0.5, tau)
        loss = loss.clone()
        loss[1] = loss[1] * 3 / B
        check((loss, rl[:3], g[:3]), ids, top, rest, s, kind, 0.5, tau, None, f"gap {gap} {kind} {dtype}")
        assert np.isfinite(host(rl)).all()
        g = topk_ref.values(host(g[:3]).reshape(3, V))
        for n in range(3):
            lim = (step + 2.0 ** -15) * 1.01 * np.abs(g[n]).sum() + 40 * LOG_SUM
            assert abs(g[n].sum()) <= lim, f"gap {gap} {kind} {dtype}: {g[n].sum()}"
            if kind == "fkl":
                e = np.exp(topk_ref.values(t[n]) - topk_ref.values(t[n]).max())
                P = np.delete(e, ids[n]).sum() / e.sum()
                assert abs(np.delete(g[n], ids[n]).sum() + P) <= lim, f"gap {gap} {dtype}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("V", [3001, 12007])
@pytest.mark.parametrize("fill", ["lowest", -1.0e4, -1.0e30])
def test_gradient_of_a_student_with_finite_fills(osd, fill, V, kind, dtype):
    """Masked tokens at a large negative number, in the record and outside it: the
    gradient as the reference has it.  (FKL's loss is up to the type's largest; the
    batch's sum of it may leave fp32.)"""
    B, k, tau = 4, 33, 1.0
    t = as_dtype(rows("normal", B, V, 6), dtype)
    ids, top, rest = record(t, k, tau)
    s = rows("normal", B, V, 7)
    g = np.random.default_rng(8)
    fill = lowest(dtype) if fill == "lowest" else np.float32(fill)
    s[0, g.random(V) < 0.9] = fill
    s[1] = fill
    s[1, ids[1]] = rows("normal", 1, k, 9)[0]          # all outside
    s[2, ids[2, : k // 2]] = fill                      # half the record
    s[3, g.random(V) < 0.5] = fill
    s[3, ids[3]] = rows("normal", 1, k, 10)[0]
    s = as_dtype(s, dtype)
    loss, rl, gr = call(osd, ids, top, rest, s, B, 1, kind, 0.5, tau)
    _, wr, wg = topk_ref.distill(ids, top, rest, s, kind, 0.5, tau)
    assert np.allclose(host(rl).reshape(-1), wr, rtol=1e-5, atol=4 * LOG_SUM)
    gr = topk_ref.values(host(gr).reshape(B, V))
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    err, lim = np.abs(gr - wg), (step + 2.0 ** -15) * np.abs(wg) + 40 * LOG_SUM * qof(s, tau) + tiny
    bad = ~(err <= lim)
    assert not bad.any(), f"{bad.sum()}: {gr[bad][:3]} for {wg[bad][:3]}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["fkl", "rkl", "jsd"])
@pytest.mark.parametrize("tau,gap", [(1.0, 88.0), (1.0, 110.0), (1.0, 600.0), (1.0, 1.0e4), (0.05, 0.0), (0.02, 0.0)])
@pytest.mark.parametrize("V", [1001, 32003])
def test_records_of_teachers_with_little_mass_outside(osd, V, tau, gap, kind, dtype):
    """osd_topk's records of rows with far peaks and at small temperatures, distilled
    from: KL(q || p) needs the logarithm of the teacher's rest, however small that is.

    The rest is within 8.4e-6 and half a step of the exact one (test_topk_gpu.py), which
    enters D through the student's Q <= 1 once and its gradient through q_j Q.  The
    others' exponentials are taken relative to their largest in 32 bits: below 2^-126 of
    it (reached at small tau) v_exp_f32 gives 0, which leaves out less than 2^-126 of the
    largest gradient."""
    tau = float(np.float32(tau))
    B, k = 4, 40
    g = np.random.default_rng(V)
    t, s = rows("normal", B, V, 90), rows("normal", B, V, 91)
    for n, peaks in enumerate((1, 5, k, 0)):
        t[n, g.choice(V, peaks, replace=False)] += np.float32(gap)
    t, s = as_dtype(t, dtype), as_dtype(s, dtype)
    ids, top, rest, _ = osd.osd_topk(to_device(t), k, tau)
    wi, wt, wrest = record(t, k, tau)
    assert np.array_equal(host(ids), wi) and np.isfinite(host(rest)).all()
    got = osd.osd_distill_topk_loss_grad(ids.view(B, 1, k), top.view(B, 1, k), rest.view(B, 1),
                                         to_device(s.reshape(B, 1, V)), kind, 0.5, tau)
    wl, wr, wg = topk_ref.distill(wi, wt, topk_ref.topk(t, k, tau)["rest"], s, kind, 0.5, tau)
    off = 8.4e-6 + 2.0 ** -24 * np.abs(wrest)
    rl = host(got[1]).reshape(-1)
    assert (np.abs(rl - wr) <= 4 * LOG_SUM + 1e-5 * np.abs(wr) + off).all(), f"{rl} {wr}"
    gr = topk_ref.values(host(got[2]).reshape(B, V))
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tiny = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    lim = ((step + 2.0 ** -15) * np.abs(wg) + (40 * LOG_SUM * np.maximum(1.0, np.abs(wr)) + 2 * off)[:, None]
           * qof(s, tau) / tau + tiny + 2.0 ** -126 * np.abs(wg).max(-1, keepdims=True))
    err = np.abs(gr - wg)
    assert (err <= lim).all(), f"{(err > lim).sum()}: {gr[err > lim][:3]} {wg[err > lim][:3]}"
