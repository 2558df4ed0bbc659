"""Builds libastraea.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a.

    python -m paper_2506_05096_b200.build [--force] [--verbose]
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libastraea.so")
SOURCES = ["api.cu", "api_operators.cu", "score.cu", "select.cu", "scatter.cu", "attn.cu", "linear.cu", "elementwise.cu", "head_norm.cu", "quantize.cu",
           "linear_fp8.cu", "linear_fp8_rows.cu"]
HEADERS = ["common.cuh", "sm100_ptx.cuh", "bounded_wait.cuh", "copy_rows.cuh", "window_keys.cuh", "linear_tiles.cuh", "epilogue_math.cuh",
           os.path.join("..", "..", "include", "astraea.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-cudart", "static"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not (force or _stale()):
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [nvcc, *NVCC_FLAGS, "-shared", "-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
