"""Build libosd.so, the HIP library behind include/osd.h, for gfx950.

Each translation unit under csrc/ is compiled by hipcc in parallel, then
linked into paper_2310_07177_amd/libosd.so (in-tree, next to the binding).
"""
import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libosd.so")
PROBE_LIB = os.path.join(HERE, "libosd_probe.so")
SOURCES = ["osd_api.hip", "verify.hip", "distill.hip", "verify_greedy.hip", "distill_stream.hip", "verify_distill.hip",
           "sample.hip", "verify_shard.hip", "verify_tree.hip", "topk.hip", "distill_topk.hip", "verify_topk.hip",
           "cache.hip", "tree_attention.hip", "tree_attention_wide_bf16.hip", "tree_attention_wide_f32.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # every rounding is the one written in the source
    "-ffp-contract=off",
    # no packed fp32 instructions (v_pk_*_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def _compile(src):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msg = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and "not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{msg}")
    return obj, msg


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        results = list(ex.map(_compile, SOURCES))
    if verbose:
        for _, msg in results:
            if msg.strip():
                print(msg, file=sys.stderr)
    objs = [o for o, _ in results]
    tmp = LIB + ".tmp"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs,
                   check=True)
    os.replace(tmp, LIB)
    # The benchmark's read-ceiling probe, a library of its own.
    probe = os.path.join(CSRC, "probe", "read_ceiling.hip")
    tmp = PROBE_LIB + ".tmp"
    r = subprocess.run([HIPCC] + FLAGS + ["-shared", "-o", tmp, probe], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {probe}:\n{r.stdout}{r.stderr}")
    os.replace(tmp, PROBE_LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
