"""Host checks of the operators on records of top logits: every mistake is
refused before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2310_07177_amd as osd

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x10004)
NAN, INF = float("nan"), float("inf")


def topk(**kw):
    a = dict(x=FAKE, stride=64, dtype=1, N=4, V=64, k=8, T=1.0, u=FAKE, ids=FAKE, top=FAKE, rest=FAKE, toks=FAKE)
    a.update(kw)
    return osd.lib().osd_topk(a["x"], a["stride"], a["dtype"], a["N"], a["V"], a["k"], a["T"], a["u"], a["ids"],
                              a["top"], a["rest"], a["toks"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), -1), (dict(ids=None), -1), (dict(top=None), -1), (dict(u=None), -1), (dict(stride=63), -1),
    (dict(N=0), -1), (dict(N=-1), -1), (dict(V=0), -1), (dict(dtype=2), -1), (dict(k=0), -1), (dict(k=-3), -1),
    (dict(k=65), -1), (dict(k=257, V=1000, stride=1000), -1),
    (dict(T=-1.0), -1), (dict(T=NAN), -1), (dict(T=INF), -1), (dict(T=0.0), -1),  # rest at T == 0
    (dict(V=1 << 20, stride=1 << 20), -2), (dict(dtype=0, V=65537, stride=65537), -2),
])
def test_topk_rejects_bad_arguments(kw, status):
    assert topk(**kw) == status


def distill(**kw):
    a = dict(ids=FAKE, top=FAKE, rest=FAKE, rows=3, k=8, s=FAKE, ss=2 * 64, dtype=1, B=2, K=2, V=64, mask=None,
             kind=0, beta=0.5, tau=1.0, loss=FAKE, row=None, grad=None, ws=FAKE, wsb=1 << 20)
    a.update(kw)
    return osd.lib().osd_distill_topk_loss_grad(
        a["ids"], a["top"], a["rest"], a["rows"], a["k"], a["s"], a["ss"], a["dtype"], a["B"], a["K"], a["V"],
        a["mask"], a["kind"], a["beta"], a["tau"], a["loss"], a["row"], a["grad"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(ids=None), -1), (dict(top=None), -1), (dict(s=None), -1), (dict(loss=None), -1),
    (dict(B=0), -1), (dict(K=0), -1), (dict(V=0), -1), (dict(B=1 << 20, K=1 << 12), -1), (dict(dtype=3), -1),
    (dict(kind=3), -1), (dict(kind=1, rest=None), -1), (dict(k=0), -1), (dict(k=65), -1), (dict(k=257, V=512), -1),
    (dict(tau=0.0), -1), (dict(tau=-1.0), -1), (dict(tau=NAN), -1), (dict(tau=INF), -1),
    (dict(beta=-0.1), -1), (dict(beta=1.1), -1), (dict(beta=NAN), -1),
    (dict(rows=1), -1), (dict(ss=127), -1),
    (dict(grad=ctypes.c_void_p(0x10002)), -1),                  # begins inside the student rows
    (dict(grad=ctypes.c_void_p(0x10000 - 2)), -1),
    (dict(grad=FAKE, ss=200), -1),                              # their own place, but rows with gaps
    (dict(V=1 << 20, ss=1 << 22), -2),
    (dict(ws=None), -4), (dict(wsb=8), -4), (dict(ws=ODD), -4),
])
def test_distill_rejects_bad_arguments(kw, status):
    assert distill(**kw) == status


def verify(**kw):
    a = dict(t=FAKE, ids=FAKE, top=FAKE, k=8, dtype=1, B=2, K=3, V=64, y=FAKE, dl=None, ua=FAKE, ur=FAKE, T=1.0,
             acc=FAKE, toks=FAKE, rmask=None, ws=FAKE, wsb=1 << 20)
    a.update(kw)
    return osd.lib().osd_verify_topk(a["t"], a["ids"], a["top"], a["k"], a["dtype"], a["B"], a["K"], a["V"], a["y"],
                                     a["dl"], a["ua"], a["ur"], a["T"], a["acc"], a["toks"], a["rmask"], a["ws"],
                                     a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=None), -1), (dict(ids=None), -1), (dict(top=None), -1), (dict(y=None), -1), (dict(ua=None), -1),
    (dict(ur=None), -1), (dict(acc=None), -1), (dict(toks=None), -1),
    (dict(B=0), -1), (dict(K=0), -1), (dict(K=17), -1), (dict(V=0), -1), (dict(dtype=9), -1),
    (dict(k=0), -1), (dict(k=65), -1), (dict(k=257, V=512), -1),
    (dict(T=0.0), -1), (dict(T=-1.0), -1), (dict(T=NAN), -1), (dict(T=INF), -1),
    (dict(V=1 << 20), -2), (dict(dtype=0, V=65537), -2),
    (dict(ws=None), -4), (dict(wsb=8), -4), (dict(ws=ODD), -4),
])
def test_verify_rejects_bad_arguments(kw, status):
    assert verify(**kw) == status


def test_workspace_sizes():
    L = osd.lib()
    for f in (L.osd_distill_topk_workspace_bytes, L.osd_verify_topk_workspace_bytes):
        assert f(0, 4) == 0 and f(4, 0) == 0 and f(-1, 1) == 0 and f(64, 8) > 0
    assert L.osd_verify_topk_workspace_bytes(4, 17) == 0


def test_binding_refuses_cpu_tensors_shapes_and_types():
    import torch
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        osd.osd_topk(x, 2)
    with pytest.raises(ValueError):
        osd.osd_topk(torch.zeros(8, 2).t(), 2)
    ids, top = torch.zeros(2, 1, 2, dtype=torch.int32), torch.zeros(2, 1, 2)
    with pytest.raises(ValueError):
        osd.osd_distill_topk_loss_grad(ids, top, None, torch.zeros(2, 1, 8), "fkl")
    with pytest.raises(ValueError):
        osd.osd_verify_topk(torch.zeros(2, 2, 8), ids, top, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1),
                            torch.zeros(2), 1.0)
