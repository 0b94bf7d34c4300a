"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libffd_b200.so")
SOURCES = [os.path.join(CSRC, f) for f in ("ffd.cu", "ffd_byte.cu", "ffd_prefix.cu")]
HEADERS = [os.path.join(CSRC, f) for f in ("ffd_kernels.cuh", "ffd_fused.cuh", "ffd_host.cuh", "ffd_own.cuh", "ffd_paged.cuh",
                                           "ffd_prefix.cuh")] + [
           os.path.join(os.path.dirname(_HERE), "include", "ffd.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads=0", "-shared",
              "-Xcompiler", "-fPIC"]


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    built = os.path.getmtime(LIB_PATH)
    return any(os.path.exists(f) and os.path.getmtime(f) > built for f in SOURCES + HEADERS)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile ``csrc/*.cu`` into ``libffd_b200.so`` next to this file (cross-compiles without a GPU)."""
    if force or is_stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = LIB_PATH + f".tmp{os.getpid()}"
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
        subprocess.check_call(cmd)
        os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
