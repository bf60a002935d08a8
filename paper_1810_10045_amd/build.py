"""Compile the HIP sources under ``csrc/`` into ``liblmzipf.so`` for gfx950, and
``csrc/calls.cpp`` into ``_lmzipf_calls.so``, the Python side of its short calls.

Every source is compiled with packed-fp32 instructions disabled
(``-target-feature -packed-fp32-ops``): the compiler would otherwise pair
fp32 adds and multiplies into packed forms on its own.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "liblmzipf.so")
CALLS_PATH = os.path.join(HERE, "_lmzipf_calls.so")
BUILD_DIR = os.path.join(HERE, "_build")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function", "-I", os.path.join(HERE, "..", "include")]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build_calls(verbose: bool = False) -> str:
    """Compile the extension module against this Python and torch (host code only)."""
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    tmp = CALLS_PATH + f".tmp{os.getpid()}"
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *(f"-I{p}" for p in (*include_paths(), sysconfig.get_paths()["include"])),
           os.path.join(CSRC, "calls.cpp"), "-o", tmp, *(f"-L{p}" for p in library_paths()),
           "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, CALLS_PATH)
    return CALLS_PATH


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library and the extension module
    (always rebuilds)."""
    os.makedirs(BUILD_DIR, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
        cmd = [HIPCC, *FLAGS, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
        return obj

    srcs = sources()
    with ThreadPoolExecutor(max(1, min(len(srcs) + 1, os.cpu_count() or 1))) as ex:
        calls = ex.submit(build_calls, verbose)
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs],
                   check=True)
    os.replace(tmp, LIB_PATH)
    calls.result()  # raises where it failed; the library does not need it
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
