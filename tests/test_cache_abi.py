"""Host checks of the operators on the paged cache: every mistake is refused
before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2310_07177_amd as osd
from paper_2310_07177_amd import binding

P = ctypes.c_void_p
FAKE, ODD = P(0x10000), P(0x10008)  # never dereferenced: every call below fails validation
NAN, INF = float("nan"), float("inf")

CACHE = dict(kc=FAKE, vc=FAKE, ps=2 * 16 * 64, pages=8, S=16, H=2, D=64, dtype=1, table=FAKE, T=4, len=FAKE)
BAD_CACHE = [
    (dict(kc=None), -1), (dict(vc=None), -1), (dict(table=None), -1), (dict(len=None), -1), (dict(kc=ODD), -1),
    (dict(vc=ODD), -1), (dict(ps=2 * 16 * 64 - 8), -1), (dict(ps=2 * 16 * 64 + 4), -1), (dict(ps=1 << 41), -1),
    (dict(pages=0), -1), (dict(pages=-1), -1), (dict(S=0), -1), (dict(H=0), -1), (dict(D=0), -1), (dict(T=0), -1),
    (dict(T=1 << 28), -1), (dict(S=1 << 26, ps=1 << 40), -1), (dict(H=70000, ps=1 << 38), -1), (dict(dtype=2), -1),
    (dict(D=60), -2), (dict(D=264, ps=1 << 20), -2), (dict(B=0), -1), (dict(N=0), -1), (dict(B=4097), -2),
]


def call(name, layout, a, fields):
    """A call's struct, in the header's order."""
    v = [a[x] for x in ("kc", "vc", "ps", "table", "len", "pages", "S", "H", "D", "dtype", "T", "B", "N") + fields]
    v = [(x.value or 0) if isinstance(x, P) else 0 if x is None else x for x in v]
    return getattr(osd.lib(), name)(layout.pack(*v), None)


def append(**kw):
    a = dict(CACHE, q=FAKE, qs=4 * 64, qo=P(0x90000), qos=4 * 64, Hq=4, k=FAKE, ks=128, v=FAKE, vs=128, B=2, N=3,
             parent=None, new=None, rot=FAKE, rows=100, R=64, style=0)
    a.update(kw)
    return call("osd_cache_append", binding._APPEND, a, ("q", "qs", "qo", "qos", "k", "ks", "v", "vs", "parent", "new", "rot",
                                                         "Hq", "rows", "R", "style"))


@pytest.mark.parametrize("kw,status", BAD_CACHE + [
    (dict(k=None), -1), (dict(v=None), -1), (dict(k=ODD), -1), (dict(v=ODD), -1), (dict(q=None), -1),
    (dict(qo=None), -1), (dict(q=ODD), -1), (dict(qo=P(0x90008)), -1), (dict(qs=248), -1), (dict(qs=260), -1),
    (dict(qos=248), -1), (dict(ks=120), -1), (dict(vs=132), -1), (dict(ks=1 << 29), -1), (dict(Hq=0), -1),
    (dict(qo=P(0x10010)), -1),                        # begins inside q
    (dict(qo=FAKE, qos=320), -1),                     # its own place, but another distance
    (dict(N=65, parent=FAKE), -1), (dict(B=4096, N=1 << 20), -1),
    (dict(R=0), -1), (dict(R=63), -1), (dict(R=66), -1), (dict(R=-2), -1), (dict(rows=0), -1), (dict(style=2), -1),
    (dict(rot=ODD), -1),
])
def test_append_rejects_bad_arguments(kw, status):
    assert append(**kw) == status


def attention(**kw):
    a = dict(CACHE, q=FAKE, qs=256, Hq=4, B=2, N=3, parent=None, new=None, scale=0.1, out=P(0x90000), ws=FAKE,
             wsb=1 << 34)
    a.update(kw)
    return call("osd_tree_attention", binding._ATTENTION, a, ("q", "qs", "parent", "new", "out", "ws", "wsb", "Hq", "scale"))


@pytest.mark.parametrize("kw,status", BAD_CACHE + [
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=ODD), -1), (dict(out=P(0x90004)), -1), (dict(qs=128), -1),
    (dict(qs=252), -1), (dict(Hq=0), -1), (dict(Hq=5), -1), (dict(N=65), -1), (dict(scale=NAN), -1),
    (dict(scale=INF), -1), (dict(scale=-INF), -1), (dict(out=FAKE), -1), (dict(out=P(0x10100)), -1),
    (dict(ws=None), -4), (dict(wsb=8), -4), (dict(ws=ODD), -4),
])
def test_attention_rejects_bad_arguments(kw, status):
    assert attention(**kw) == status


def keep(**kw):
    a = dict(CACHE, layers=2, ls=1 << 20, B=2, N=3, path=FAKE, acc=FAKE, new=P(0x90000), reserved=0)
    a.update(kw)
    return call("osd_cache_keep", binding._KEEP, a, ("ls", "path", "acc", "new", "layers", "reserved"))


@pytest.mark.parametrize("kw,status", BAD_CACHE + [
    (dict(path=None), -1), (dict(acc=None), -1), (dict(new=None), -1), (dict(new=FAKE), -1), (dict(new=P(0x10004)), -1),
    (dict(N=65), -1), (dict(layers=0), -1), (dict(layers=70000), -1), (dict(ls=-8), -1), (dict(ls=4), -1),
    (dict(ls=1 << 41), -1),
])
def test_keep_rejects_bad_arguments(kw, status):
    assert keep(**kw) == status


def test_no_call_is_refused():
    L = osd.lib()
    assert L.osd_cache_append(None, None) == L.osd_tree_attention(None, None) == L.osd_cache_keep(None, None) == -1


def test_structs_are_the_headers(tmp_path):
    """The binding packs the structs as C lays them out."""
    import os
    import subprocess
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "osd.h"\nint main(void) { printf("%zu %zu %zu", sizeof(osd_append), '
                   'sizeof(osd_attention), sizeof(osd_keep)); return 0; }\n')
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [binding._APPEND.size, binding._ATTENTION.size, binding._KEEP.size]


def test_workspace_sizes():
    f = osd.lib().osd_tree_attention_workspace_bytes
    assert f(4, 8, 32, 8, 128) > 0 and f(4096, 64, 64, 8, 256) > 0
    for a in ((0, 8, 32, 8, 128), (4097, 8, 32, 8, 128), (4, 0, 32, 8, 128), (4, 65, 32, 8, 128), (4, 8, 0, 8, 128),
              (4, 8, 32, 0, 128), (4, 8, 33, 8, 128), (4, 8, 32, 8, 100), (4, 8, 32, 8, 264)):
        assert f(*a) == 0


def test_binding_refuses_shapes_types_and_cpu_tensors():
    import torch
    i32 = dict(dtype=torch.int32)
    kc = torch.zeros(4, 2, 16, 64)
    table, length = torch.zeros(1, 2, **i32), torch.zeros(1, **i32)
    k, q = torch.zeros(1, 3, 2, 64), torch.zeros(1, 3, 4, 64)
    path, acc = torch.zeros(1, 3, **i32), torch.zeros(1, **i32)
    for call in (lambda: osd.osd_cache_append(k, k, kc, kc, table, length),                  # CPU
                 lambda: osd.osd_tree_attention(q, kc, kc, table, length),
                 lambda: osd.osd_cache_keep(kc, kc, table, length, path, acc),
                 lambda: osd.osd_tree_attention(q, kc, kc[:2], table, length),               # shapes
                 lambda: osd.osd_tree_attention(q, kc.transpose(1, 2), kc.transpose(1, 2), table, length),
                 lambda: osd.osd_tree_attention(q, kc, kc, table.long(), length),
                 lambda: osd.osd_tree_attention(q, kc, kc, table, torch.zeros(2, **i32)),
                 lambda: osd.osd_cache_keep(kc, kc, table, length, path[0], acc),
                 lambda: osd.osd_cache_keep(kc[0], kc[0], table, length, path, acc)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        osd.osd_tree_attention(q, kc, kc.bfloat16(), table, length)
    with pytest.raises(TypeError):
        osd.osd_tree_attention(q.half(), kc.half(), kc.half(), table, length)


def test_binding_refuses_distances_that_are_not_one():
    import torch
    f = lambda t: binding._token_stride(t, *t.shape, t.dtype, "q")
    x = torch.zeros(2, 3, 8, 64)
    assert f(x) == 512 and f(x[:, :, 2:4]) == 512 and f(x[:, :1, :4]) == 3 * 512
    for t in (x[:, :2], x.transpose(1, 2), x[..., ::2], x[:, :, ::2]):
        with pytest.raises(ValueError):
            f(t)
