"""Two host threads that call an operator of several launches on one stream and
one workspace: the launches of a call stay together, so that what one of them
leaves in the workspace for the next is not another call's.

No GPU: a library loaded before libosd.so stands in for hipLaunchKernel.  It
notes the thread of each launch and dwells in it, so that launches that are not
kept together interleave."""
import os
import subprocess
import sys

import pytest

from paper_2310_07177_amd import binding

STUB = r"""
#include <pthread.h>
#include <stdint.h>
#include <unistd.h>
struct dim { uint32_t x, y, z; };
static unsigned long launches[64];
static int n;
extern "C" int hipLaunchKernel(const void*, dim, dim, void**, size_t, void*) {
    const int at = __atomic_fetch_add(&n, 1, __ATOMIC_SEQ_CST);
    if (at < 64) launches[at] = (unsigned long)pthread_self();
    usleep(30000);
    return 0;
}
extern "C" int launch(int at) {  // the thread of a launch, numbered by first appearance; -1: no such launch
    if (at >= n || at >= 64) return -1;
    int id = 0;
    for (int i = 0; i < at; ++i) {
        bool first = true;
        for (int j = 0; j < i; ++j) first = first && launches[j] != launches[i];
        if (launches[i] == launches[at]) break;
        id += first;
    }
    return id;
}
"""

CALLS = r"""
import ctypes, sys, threading
stub = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
L = ctypes.CDLL(sys.argv[2])
p = lambda x: ctypes.c_void_p(x)  # never read: nothing is launched
f = ctypes.c_float
L.osd_distill_topk_workspace_bytes.restype = L.osd_verify_distill_workspace_bytes.restype = ctypes.c_size_t

def distill_topk(grad):
    B, K, V, k = 4, 1, 128256, 64
    n = ctypes.c_size_t(L.osd_distill_topk_workspace_bytes(B, K))
    return L.osd_distill_topk_loss_grad(p(0x10000), p(0x10000), p(0x10000), ctypes.c_int64(K), k, p(0x1000000),
                                        ctypes.c_int64(K * V), 1, B, K, V, None, 0, f(0.5), f(1.0), p(0x10000), None,
                                        p(0x8000000) if grad else None, p(0x20000), n, None)

def verify_distill_rejected():
    B, K, V = 4, 2, 5
    n = ctypes.c_size_t(L.osd_verify_distill_workspace_bytes(B, K))
    return L.osd_verify_distill_rejected(p(0x1000000), p(0x2000000), 1, B, K, V, p(0x10000), None, p(0x10000),
                                         p(0x10000), f(1.0), p(0x10000), p(0x10000), None, 0, f(0.5), p(0x10000),
                                         None, None, p(0x20000), n, None)

call = {"distill_topk": lambda: distill_topk(False), "distill_topk_grad": lambda: distill_topk(True),
        "verify_distill_rejected": verify_distill_rejected}[sys.argv[3]]
start, status = threading.Barrier(2), [None, None]

def thread(i):
    start.wait()
    status[i] = call()

threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
[t.start() for t in threads]
[t.join() for t in threads]
assert status == [0, 0], status
order = []
while stub.launch(len(order)) >= 0:
    order.append(stub.launch(len(order)))
print("launches", *order)
"""


@pytest.mark.parametrize("call,each", [("distill_topk", 2), ("distill_topk_grad", 2),
                                       ("verify_distill_rejected", 3)])
def test_launches_of_a_call_stay_together(call, each, tmp_path):
    stub = str(tmp_path / "stub.so")
    (tmp_path / "stub.cpp").write_text(STUB)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-o", stub, str(tmp_path / "stub.cpp"), "-lpthread"], check=True)
    r = subprocess.run([sys.executable, "-c", CALLS, stub, binding.LIB_PATH, call], capture_output=True, text=True,
                       timeout=120, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr[-2000:]
    order = [int(x) for x in r.stdout.split("launches")[1].split()]
    assert order == [0] * each + [1] * each
