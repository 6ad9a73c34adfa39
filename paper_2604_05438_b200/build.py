"""Builds libtkphi.so (the C-ABI library) in-tree with nvcc for sm_100a, and the CPython module of the paged calls."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtkphi.so")
SOURCES = ["api.cu", "score.cu", "select_cluster.cu", "exact_residual.cu", "build_summaries.cu", "static_scratch.cu",
           "selftest.cu", "cached_features.cu",
           "mlp_features.cu", "mlp_query.cu", "paged_api.cu", "paged_append.cu", "paged_rows.cu",
           "paged_tiles.cu", "paged_select.cu"]
HEADERS = ["common.cuh", "sm100.cuh", "feature_jobs.cuh", "host.cuh", "paged.cuh", os.path.join("..", "..", "include", "tkphi.h")]


BINDING = os.path.join(HERE, "_paged_binding.so")
BINDING_SOURCE = os.path.join(CSRC, "paged_binding.cpp")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def needs_build() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(BINDING):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(BINDING))
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [BINDING_SOURCE, os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every kernel for sm_100a into one shared library; returns its path."""
    if not force and not needs_build():
        return LIB
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-DNDEBUG",
           "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libtkphi.so")
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    build_binding(verbose)
    return LIB


def build_binding(verbose: bool = False) -> str:
    """Compile the CPython module of the paged calls against torch's headers and libtkphi.so; returns its path."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    include = [sysconfig.get_paths()["include"], os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-DNDEBUG",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-o", BINDING, BINDING_SOURCE]
    cmd += [f"-I{d}" for d in include]
    cmd += [f"-L{HERE}", "-l:libtkphi.so", "-Wl,-rpath,$ORIGIN", f"-L{os.path.join(root, 'lib')}",
            f"-Wl,-rpath,{os.path.join(root, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("the C++ compiler failed building _paged_binding.so")
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    return BINDING


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
