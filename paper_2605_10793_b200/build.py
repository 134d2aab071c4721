"""Build libconqur.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libconqur.so")
OBJ = os.path.join(PKG, "build")
SOURCES = ["conqur.cu", "conqur_noalloc.cu", "conqur_heads.cu", "conqur_kv.cu"]
HEADERS = ["conqur_internal.h", "conqur_simt.cuh", "conqur_ptx.cuh", "conqur_tc.cuh", "conqur_tc_batched.cuh", "conqur_split_tc.cuh", "conqur_ns_cluster.cuh", "conqur_fold_tc.cuh", "conqur_aux.cuh", "conqur_hadamard_tc.cuh", "conqur_attention.cuh", "conqur_attention_tc.cuh", "ns_schedule.h",
           os.path.join("..", "..", "include", "conqur.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    return any(os.path.getmtime(p) > t for p in deps if os.path.exists(p))


def _nvcc(args) -> str:
    nvcc = os.environ.get("NVCC", "nvcc")
    res = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a"] + args, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libconqur.so")
    return res.stderr


def build(force: bool = False, verbose: bool = False, only=None) -> str:
    """Compile every source (side by side) and link.  only: compile just these sources, taking the other objects as they are."""
    if not force and not only and not _stale():
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    objects = {s: os.path.join(OBJ, s + ".o") for s in SOURCES}
    flags = ["-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-diag-suppress", "177"] + (["-Xptxas", "-v"] if verbose else [])
    todo = [s for s in SOURCES if not only or s in only or not os.path.exists(objects[s])]
    with ThreadPoolExecutor(len(todo)) as pool:
        said = list(pool.map(lambda s: _nvcc(flags + ["-c", "-o", objects[s], os.path.join(CSRC, s)]), todo))
    if verbose:
        sys.stderr.write("".join(said))
    _nvcc(["-shared", "-o", LIB] + list(objects.values()))
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, only=[a for a in sys.argv[1:] if a.endswith(".cu")]))
