"""Builds the CUDA library in-tree with nvcc for sm_100a, and with g++ the module that marshals the cache's calls (no JIT cache)."""
from __future__ import annotations

import os
import subprocess
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libbv_b200.so")
SOURCES = ["bv_api.cu", "bv_stream.cu", "bv_cluster.cu", "bv_flow.cu", "bv_small.cu", "bv_phase.cu", "bv_noalloc.cu", "bv_sample.cu", "bv_loop.cu",
           "bv_cache.cu", "bv_attend_rows.cu", "bv_attend_tiles.cu", "bv_pages.cu", "bv_rotary.cu", "bv_prompt.cu", "bv_prompt_tiles.cu", "bv_filter.cu"]
HEADERS = ["bv_device.cuh", "bv_launch.h", "bv_flow_common.cuh", "bv_sample_row.cuh", "bv_cache.cuh", "bv_tensor.cuh", "bv_prompt.cuh", os.path.join("..", "..", "include", "bv.h")]

FAST_SOURCE = os.path.join(CSRC, "fast.cpp")
FAST_PATH = os.path.join(_HERE, "_fast.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
]


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libbv_b200.so next to this file; returns its path."""
    if force or _stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        tmp = LIB_PATH + ".%d.tmp" % os.getpid()
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
              [os.path.join(CSRC, f) for f in SOURCES] + ["-o", tmp]
        subprocess.check_call(cmd)
        os.replace(tmp, LIB_PATH)
    build_fast(force)
    return LIB_PATH


def build_fast(force: bool = False) -> str:
    """Compile csrc/fast.cpp into the module _fast next to this file (plain C++ on torch's and CUDA's headers); returns its path."""
    header = os.path.join(CSRC, "..", "..", "include", "bv.h")
    if force or not os.path.exists(FAST_PATH) or os.path.getmtime(FAST_PATH) < max(os.path.getmtime(FAST_SOURCE), os.path.getmtime(header)):
        import torch
        root = os.path.dirname(torch.__file__)
        cuda = os.path.join(os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))), "include")
        tmp = FAST_PATH + ".%d.tmp" % os.getpid()
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
                               "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"),
                               "-I" + sysconfig.get_paths()["include"], "-I" + cuda, FAST_SOURCE, "-o", tmp,
                               "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])
        os.replace(tmp, FAST_PATH)
    return FAST_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
