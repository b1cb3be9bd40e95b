"""Build ``libcconv.so`` (the C-ABI library) in-tree with nvcc for sm_100a.

Usage: ``python -m paper_1802_06905_b200.build [--force] [--verbose]``.
The CUDA runtime is linked statically and the driver API is resolved at run time, so the library
loads (and its host-only entry points work) on a machine without a GPU.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcconv.so")
SOURCES = ["kernels.cu", "direct_kernel.cu", "stem_kernel.cu", "api.cu", "host_setup.cu", "noalloc.cu", "pool.cu", "planner.cpp",
           "block_api.cu", "block_few.cu", "block_ffn.cu", "block_fp8.cu", "block_gemm.cu", "block_tma.cu", "block_norm.cu", "block_quant.cu"]
HEADERS = ["kernels.h", "planner.h", "host_setup.h", "ptx_sm100.cuh", "direct_issue.cuh",
           "block.h", "block_device.cuh", "block_few.h", "block_ffn.h", "block_fp8.h", "block_launch.h", "block_steps.h", "block_gemm.h", "block_tma.h", "pair_sm100.cuh", "block_norm.h", "block_quant.h",
           os.path.join("..", "..", "include", "cconv_block.h"), os.path.join("..", "..", "include", "cconv.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every source to an object file (in parallel, only those older than a source or
    header) and link the shared library."""
    if not force and not needs_build():
        return LIB
    from concurrent.futures import ThreadPoolExecutor
    objdir = os.path.join(HERE, "build")
    os.makedirs(objdir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "-Xcompiler", "-fPIC"]
    if verbose:
        flags += ["-Xptxas", "-v"]
    newest_header = max(os.path.getmtime(os.path.join(CSRC, h)) for h in HEADERS)

    def compile_one(src: str) -> str:
        path = os.path.join(CSRC, src)
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        stale = (force or not os.path.exists(obj)
                 or os.path.getmtime(obj) < max(os.path.getmtime(path), newest_header))
        if stale:
            subprocess.run([_nvcc(), *flags, "-c", path, "-o", obj], check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 4)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    subprocess.run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart",
                    "static", "-o", LIB, *objs], check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
