"""Builds libfastkv_b200.so (hand-written CUDA for sm_100a behind a C ABI) in-tree with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libfastkv_b200.so")
SOURCES = ["api.cu", "score.cu", "score_fused.cu", "score_parked.cu", "select.cu", "compact.cu", "decode_attn.cu", "score_static.cu", "prefill_attn.cu", "paged_append.cu",
           "paged_attn.cu", "paged_weights.cu", "paged_evict.cu", "prefix_attn.cu"]
HEADERS = ["common.cuh", "score.cuh", "select.cuh", "compact.cuh", "decode_attn.cuh", "prefill_attn.cuh", "paged.cuh", "paged_index.h", "paged_mma.cuh",
           os.path.join("..", "..", "include", "fastkv.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--shared"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("nvcc not found")


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source of the package for sm_100a into one shared library."""
    if not force and not is_stale():
        return LIB_PATH
    tmp = LIB_PATH + ".tmp%d" % os.getpid()
    cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
        [os.path.join(CSRC, f) for f in SOURCES] + ["-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
