"""Compile the CUDA library (sm_100a only) in-tree: paper_2302_01318_b200/libsps_b200.so."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsps_b200.so")
SOURCES = ["engine.cu", "linear.cu", "linear_tc.cu", "attention.cu", "sampler.cu", "wide.cu", "tp.cu", "paged.cu", "paged_attention.cu", "paged_attention_tc.cu", "paged_attention_wide.cu", "pages.cu", "beam.cu"]
HEADERS = ["common.cuh", "paged.cuh", "paged_tc.cuh", os.path.join("..", "..", "include", "sps.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
              "-shared"]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        extra = os.environ.get("SPS_NVCC_EXTRA", "").split()   # e.g. -D switches of a debugging build
        cmd = [nvcc] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
