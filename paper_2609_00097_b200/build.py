"""Builds the CUDA library in-tree with nvcc for sm_100a (no JIT cache, no torch extension machinery), and the Python module
that checks torch tensors and calls it."""
from __future__ import annotations

import importlib.metadata
import os
import subprocess
import sysconfig
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libffd_b200.so")
SOURCES = [os.path.join(CSRC, f) for f in ("ffd.cu", "ffd_byte.cu", "ffd_prefix.cu")]
HEADERS = [os.path.join(CSRC, f) for f in ("ffd_kernels.cuh", "ffd_fused.cuh", "ffd_host.cuh", "ffd_own.cuh", "ffd_paged.cuh",
                                           "ffd_prefix.cuh", "ffd_prefix_step.cuh")] + [
           os.path.join(os.path.dirname(_HERE), "include", "ffd.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads=0", "-shared",
              "-Xcompiler", "-fPIC"]


def _torch_version() -> str:
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return "none"


# compiled against one version of torch, of which the name speaks: another one has its own
BINDING_PATH = os.path.join(_HERE, f"_ffd_binding.torch-{_torch_version()}{sysconfig.get_config_var('EXT_SUFFIX')}")
BINDING_SOURCES = [os.path.join(CSRC, "ffd_binding.cpp"), HEADERS[-1]]


def _older(path, sources) -> bool:
    if not os.path.exists(path):
        return True
    built = os.path.getmtime(path)
    return any(os.path.exists(f) and os.path.getmtime(f) > built for f in sources)


def is_stale() -> bool:
    return _older(LIB_PATH, SOURCES + HEADERS) or _older(BINDING_PATH, BINDING_SOURCES)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile ``csrc/*.cu`` into ``libffd_b200.so`` next to this file (cross-compiles without a GPU), and the binding.

    The library needs nvcc only.  Where the binding cannot be built (no C++ compiler, no headers of Python or torch) there is a
    warning, and the functions that go through it raise ImportError."""
    if force or _older(LIB_PATH, SOURCES + HEADERS):
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = LIB_PATH + f".tmp{os.getpid()}"
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
        subprocess.check_call(cmd)
        os.replace(tmp, LIB_PATH)
    try:
        build_binding(force)
    except (ImportError, OSError, subprocess.CalledProcessError) as e:
        warnings.warn(f"the binding of the byte cache and the shared prefix was not built: {e}", RuntimeWarning, stacklevel=2)
    return LIB_PATH


def build_binding(force: bool = False) -> str:
    """Compile ``csrc/ffd_binding.cpp`` against the installed torch."""
    if force or _older(BINDING_PATH, BINDING_SOURCES):
        try:
            _compile_binding()
        except BaseException:
            if os.path.exists(BINDING_PATH):      # not to be taken for the new one
                os.remove(BINDING_PATH)
            raise
    return BINDING_PATH


def _compile_binding() -> None:
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    include = [sysconfig.get_paths()["include"], os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    tmp = BINDING_PATH + f".tmp{os.getpid()}"
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *["-I" + i for i in include],
                           "-o", tmp, BINDING_SOURCES[0], "-L" + os.path.join(root, "lib"),
                           "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"])
    os.replace(tmp, BINDING_PATH)


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
