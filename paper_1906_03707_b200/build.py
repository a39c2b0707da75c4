"""Builds the C-ABI shared library in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhag_b200.so")
SOURCES = ["hag_build.cpp", "hag_cuda.cu", "hag_pool.cu", "hag_max.cu", "hag_embed.cu", "hag_norm.cu", "hag_clip.cu"]
HEADERS = [os.path.join(ROOT, "include", "hag.h"), os.path.join(CSRC, "hag_internal.h"),
           os.path.join(CSRC, "hag_kernels.cuh"), os.path.join(CSRC, "hag_launch.h"), os.path.join(CSRC, "hag_rows.cuh")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(p) > built for p in deps if os.path.exists(p))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library if it is missing or older than its sources."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    common = [nvcc, "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-gencode", "arch=compute_100a,code=sm_100a"]
    flags = ["-lineinfo", "-I", os.path.join(ROOT, "include"), "-I", CSRC] + (["-Xptxas", "-v"] if verbose else [])
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        list(pool.map(lambda p: subprocess.check_call(common + flags + ["-c", "-o", p[1], os.path.join(CSRC, p[0])]), zip(SOURCES, objects)))
        linked = f"{os.path.splitext(LIB)[0]}.{os.getpid()}.so"      # beside the library, whose place it takes in one step: a process
        try:                                                         # that has the old file mapped keeps it
            subprocess.check_call(common + ["-shared", "-o", linked] + objects + ["-ldl"])     # -ldl: the header-only NVTX ranges load their tool lazily
            os.replace(linked, LIB)
        finally:
            if os.path.exists(linked):
                os.remove(linked)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
