"""osd_topk against the 64-bit reference: ids, logits and tokens exactly (the
draws are decided in fp64), the mass outside to fp32 rounding."""
import numpy as np
import pytest

from oracle import topk_ref
from tests._helpers import to_device
from tests._topk_helpers import LOG_SUM, as_dtype, rows, uniforms

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def osd():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU")
    import paper_2310_07177_amd as m
    m.lib()
    return m


def host(t):
    import torch
    if t is None:
        return None
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


def check(got, x, k, T, u, label):
    want = topk_ref.topk(x, k, T, u)
    ids, top, rest, toks = (host(t) for t in got)
    assert np.array_equal(ids, want["ids"]), f"{label}: ids, first row {np.argwhere(ids != want['ids'])[0]}"
    assert np.array_equal(topk_ref.values(top), want["top"] + 0.0), f"{label}: logits"
    if rest is not None:
        bad = np.isneginf(rest) != np.isneginf(want["rest"])
        assert not bad.any(), f"{label}: rest {rest[bad]} {want['rest'][bad]}"
        some = ~np.isneginf(rest)
        err = np.abs(rest[some] - want["rest"][some])
        # the sum's logarithm, and the result's own rounding (half a step)
        assert (err <= LOG_SUM + 2.0 ** -24 * np.abs(want["rest"][some])).all(), f"{label}: rest off by {err.max()}"
    if toks is not None:
        sure = want["margin"] > 1e-9
        assert np.array_equal(toks[sure], want["tokens"][sure]), f"{label}: tokens"
        return int((~sure).sum())
    return 0


SHAPES = [  # V, k: every tile, odd and ragged sizes, one token, whole rows
    (1, 1), (2, 2), (7, 3), (8, 8), (9, 4), (64, 64), (100, 1), (255, 256 - 1), (1000, 63), (1001, 64), (2048, 65),
    (4099, 256), (8192, 7), (16384, 256), (20011, 33), (32000, 64), (32128, 128), (32771, 5),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", SHAPES)
def test_shapes(osd, V, k, dtype):
    N, T = 5, 0.75
    x, u = as_dtype(rows("normal", N, V, V + k), dtype), uniforms(N, V)
    unsure = check(osd.osd_topk(to_device(x), k, T, to_device(u)), x, k, T, u, f"V={V} k={k} {dtype}")
    assert unsure <= 1


@pytest.mark.parametrize("V,k,dtype", [(65536, 100, "f32"), (50257, 20, "f32"), (131072, 256, "bf16"),
                                       (128256, 64, "bf16"), (100003, 17, "bf16"), (65535, 255, "bf16")])
def test_long_rows(osd, V, k, dtype):
    N, T = 3, 1.0
    x, u = as_dtype(rows("normal", N, V, V), dtype), uniforms(N, V)
    check(osd.osd_topk(to_device(x), k, T, to_device(u)), x, k, T, u, f"V={V} k={k} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["ties", "equal", "zeros", "lowest", "masked", "masked_lowest", "ascending",
                                  "descending", "block", "peak", "wide", "bad"])
@pytest.mark.parametrize("V,k", [(1003, 37), (32000, 64), (70001, 256)])
def test_kinds(osd, kind, V, k, dtype):
    if dtype == "f32" and V > 65536:
        V = 60001
    N, T = 5, 1.0
    x, u = as_dtype(rows(kind, N, V, 11, dtype), dtype), uniforms(N, 12)
    u[0] = 0.0
    u[1] = np.float32(1.0 - 2.0 ** -24)
    check(osd.osd_topk(to_device(x), k, T, to_device(u)), x, k, T, u, f"{kind} V={V} k={k} {dtype}")


@pytest.mark.parametrize("N", [1, 2, 40, 300, 1500])
@pytest.mark.parametrize("dtype,V", [("bf16", 32003), ("f32", 9001), ("bf16", 12001), ("bf16", 50257), ("f32", 40009)])
def test_row_counts(osd, N, dtype, V):
    """Few rows and many: each row's record is its own, whatever form is launched."""
    import torch
    k, T = 50, 1.0
    x, u = as_dtype(rows("normal", min(N, 40), V, N), dtype), uniforms(N, N)
    x = np.concatenate([x] * ((N + 39) // 40))[:N]
    got = osd.osd_topk(to_device(x), k, T, to_device(u))
    one = min(N, 40)
    check([t[:one].contiguous() for t in got], x[:one], k, T, u[:one], f"N={N}")
    assert all(torch.equal(t[r], t[r - 40]) for t in got[:3] for r in range(40, N, 97))


def test_strided_rows_offsets_and_given_outputs(osd):
    """One position of every sequence, rows on odd addresses, and outputs in
    place."""
    import torch
    B, K, V, k = 6, 3, 1001, 10
    for dtype in ("bf16", "f32"):
        x = as_dtype(rows("normal", B * K, V, 21), dtype).reshape(B, K, V)
        d, u = to_device(x), uniforms(B, 22)
        out = (torch.empty(B, k, dtype=torch.int32, device="cuda"), torch.empty(B, k, dtype=d.dtype, device="cuda"),
               torch.empty(B, dtype=torch.float32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda"))
        got = osd.osd_topk(d[:, 1, :], k, 1.0, to_device(u), out=out)
        assert all(a is b for a, b in zip(got, out))
        check(got, x[:, 1], k, 1.0, u, f"strided {dtype}")


def test_greedy_and_optional_outputs(osd):
    x, u = as_dtype(rows("ties", 4, 500, 31), "bf16"), uniforms(4, 32)
    d = to_device(x)
    ids, top, rest, toks = osd.osd_topk(d, 3, 0.0, rest=False, tokens=True)
    assert rest is None and np.array_equal(host(toks), topk_ref.topk(x, 3, 0.0)["tokens"])
    assert osd.osd_topk(d, 3, 0.0, rest=False)[3] is None
    ids2, top2, rest2, toks2 = osd.osd_topk(d, 3, 1.0, to_device(u), rest=False)
    assert rest2 is None and np.array_equal(host(ids2), host(ids))
    with pytest.raises(osd.OsdError):
        osd.osd_topk(d, 3, 0.0)  # rest at T == 0
    with pytest.raises(osd.OsdError):
        osd.osd_topk(d, 257, 1.0)
    with pytest.raises(osd.OsdError):
        osd.osd_topk(d, 3, 1.0, tokens=True)  # a draw without uniforms


def test_guard_bands(osd):
    """Nothing is written outside the outputs."""
    import ctypes
    import torch
    from paper_2310_07177_amd import binding
    for N, V, k, dtype in [(3, 7, 5, "bf16"), (2, 1001, 33, "f32"), (5, 32003, 255, "bf16"), (1, 70001, 64, "bf16")]:
        x = to_device(as_dtype(rows("normal", N, V, 41), dtype))
        es = x.element_size()
        sizes = [N * k * 4, N * k * es, N * 4, N * 4]
        bufs = [torch.full((n + 8192,), 0x5A, dtype=torch.uint8, device="cuda") for n in sizes]
        u = to_device(uniforms(N, 42))
        st = osd.lib().osd_topk(ctypes.c_void_p(x.data_ptr()), V, binding.OSD_BF16 if es == 2 else binding.OSD_F32, N,
                                V, k, 1.0, ctypes.c_void_p(u.data_ptr()),
                                *(ctypes.c_void_p(b.data_ptr() + 4096) for b in bufs), None)
        assert st == 0
        torch.cuda.synchronize()
        for b, n in zip(bufs, sizes):
            assert (b[:4096] == 0x5A).all() and (b[4096 + n:] == 0x5A).all()


def test_other_stream_and_graph(osd):
    """A call on a side stream, and a captured one replayed with new inputs
    between eager calls."""
    import torch
    V, k, N, T = 32003, 64, 7, 1.0
    xs = [as_dtype(rows("normal", N, V, 50 + i), "bf16") for i in range(3)]
    us = [uniforms(N, 60 + i) for i in range(3)]
    x, u = to_device(xs[0]), to_device(us[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = osd.osd_topk(x, k, T, u)
    side.synchronize()
    check(got, xs[0], k, T, us[0], "stream")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = osd.osd_topk(x, k, T, u)
    for i in (1, 2, 0, 1):
        x.copy_(to_device(xs[i]))
        u.copy_(to_device(us[i]))
        eager = osd.osd_topk(x, k, T, u)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(out, xs[i], k, T, us[i], f"replay {i}")
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


# The others' mass where it lies far below the largest logit, or T is small: terms up
# to 100 octaves above a thread's reference (the kernel's own limit), each off by
# (2 * 100 ln 2 + 2) 2^-24 at most.
FAR_SUM = (200 * np.log(2) + 2) * 2.0 ** -24


def check_far(got, x, k, T, label):
    want = topk_ref.topk(x, k, T)
    ids, _, rest, _ = (host(t) for t in got)
    assert np.array_equal(ids, want["ids"]), f"{label}: ids"
    bad = np.isneginf(rest) != np.isneginf(want["rest"])
    assert not bad.any(), f"{label}: rest {rest[bad]} {want['rest'][bad]}"
    some = ~np.isneginf(rest)
    err = np.abs(rest[some] - want["rest"][some])
    lim = FAR_SUM + 2.0 ** -24 * np.abs(want["rest"][some])
    assert (err <= lim).all(), f"{label}: rest {rest[some][err > lim][:3]} {want['rest'][some][err > lim][:3]}"


FAR_SHAPES = [(100, 64, "f32"), (1000, 64, "bf16"), (1000, 1, "f32"), (4099, 200, "bf16"), (32000, 64, "bf16"),
              (32003, 256, "f32"), (70001, 100, "bf16"), (128256, 128, "bf16")]


@pytest.mark.parametrize("gap", [60.0, 80.0, 88.0, 95.0, 110.0, 200.0, 600.0, 1.0e4])
@pytest.mark.parametrize("V,k,dtype", FAR_SHAPES)
def test_mass_far_below_the_record(osd, V, k, dtype, gap):
    """Peaks of one token, half the record and all of it above the others; one
    row with nothing outside."""
    x = rows("normal", 4, V, 71)
    g = np.random.default_rng(72)
    for n, peaks in enumerate((1, max(1, k // 2), k)):
        x[n, g.choice(V, peaks, replace=False)] += np.float32(gap)
    keep = g.choice(V, max(1, k // 2), replace=False)
    only = np.full(V, -np.inf, np.float32)
    only[keep] = x[3, keep]
    x[3] = only
    x = as_dtype(x, dtype)
    check_far(osd.osd_topk(to_device(x), k, 1.0), x, k, 1.0, f"V={V} k={k} {dtype} gap={gap}")


@pytest.mark.parametrize("T", [0.25, 0.1, 0.05, 0.03125, 0.02, 0.001])
@pytest.mark.parametrize("V,k,dtype", FAR_SHAPES)
def test_mass_at_small_temperatures(osd, V, k, dtype, T):
    T = float(np.float32(T))
    x = as_dtype(rows("normal", 5, V, 73), dtype)
    check_far(osd.osd_topk(to_device(x), k, T), x, k, T, f"V={V} k={k} {dtype} T={T}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,N", [(1003, 3), (32000, 3), (32000, 600)])
def test_ties_far_below_the_record(osd, V, N, dtype):
    """The record's last slots and the mass outside of one value, far below the
    first slots: ids decide which of them are outside."""
    k = 40
    x = np.full((3, V), -300.0, np.float32)
    x[0, 7] = 1.0
    x[1, [3, V - 1]] = 2.0
    x[2, V // 2] = 0.5
    x[2, : V // 3] = -301.0
    x = as_dtype(x, dtype)
    got = osd.osd_topk(to_device(np.concatenate([x] * (N // 3))), k, 1.0)
    check_far([None if t is None else t[:3].contiguous() for t in got], x, k, 1.0, f"V={V} {dtype}")
    assert all((host(t)[:3] == host(t)[-3:]).all() for t in got[:3])


@pytest.mark.parametrize("N,V,k,dtype", [(4, 2, 1, "bf16"), (4, 5, 2, "bf16"), (4, 3, 2, "f32"), (4, 9, 4, "bf16"),
                                         (4, 257, 256, "f32"), (300, 128256, 64, "bf16"), (300, 65536, 256, "f32")])
def test_mass_far_below_in_short_rows_and_many_long_ones(osd, N, V, k, dtype):
    x = rows("normal", 4, V, 81)
    for n, gap in enumerate((90.0, 700.0, 3.0e4)):
        x[n, np.argsort(-x[n])[:k]] += np.float32(gap)
    x = as_dtype(x, dtype)
    got = osd.osd_topk(to_device(np.concatenate([x] * (N // 4))), k, 1.0)
    check_far([None if t is None else t[:4].contiguous() for t in got], x, k, 1.0, f"V={V} k={k} {dtype}")
    assert all((host(t)[:4] == host(t)[-4:]).all() for t in got[:3])
