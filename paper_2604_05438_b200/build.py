"""Builds libtkphi.so (the C-ABI library) in-tree with nvcc for sm_100a, and the CPython module of the paged calls."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtkphi.so")
SOURCES = ["api.cu", "score.cu", "select_cluster.cu", "exact_residual.cu", "build_summaries.cu", "static_scratch.cu",
           "selftest.cu", "cached_features.cu",
           "mlp_features.cu", "mlp_query.cu", "paged_api.cu", "paged_append.cu", "paged_rows.cu",
           "paged_tiles.cu", "paged_select.cu", "paged_write.cu", "paged_read.cu", "paged8_rows.cu"]
HEADERS = ["common.cuh", "sm100.cuh", "feature_jobs.cuh", "host.cuh", "paged.cuh", "paged_walk.cuh", "held8.cuh",
           os.path.join("..", "..", "include", "tkphi.h")]


BINDING = os.path.join(HERE, "_paged_binding.so")
BINDING_SOURCE = os.path.join(CSRC, "paged_binding.cpp")


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(built: str, deps) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(d) > os.path.getmtime(built) for d in deps)


def _torch_root() -> str:
    import torch
    return os.path.dirname(torch.__file__)


def library_needs_build() -> bool:
    return _stale(LIB, [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)])


def binding_needs_build() -> bool:
    # (another torch is another C++ interface: its version file is newer than what was built against the one before)
    return _stale(BINDING, [BINDING_SOURCE, os.path.join(CSRC, "..", "..", "include", "tkphi.h"), os.path.abspath(__file__),
                            os.path.join(_torch_root(), "version.py")])


def needs_build() -> bool:
    return library_needs_build() or binding_needs_build()


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every kernel for sm_100a into one shared library; returns its path.  The CPython module of the paged calls is
    built with it; where that fails (no C++ compiler, no torch headers) there is a warning, and the paged calls of the
    Python package raise until build_binding() succeeds: the library and everything else do not need it."""
    if force or library_needs_build():
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
    if force or binding_needs_build():
        try:
            build_binding(verbose)
        except (RuntimeError, OSError) as e:
            warnings.warn(f"libtkphi.so is built, but not the module of the paged calls: {e}")
    return LIB


def build_binding(verbose: bool = False) -> str:
    """Compile the CPython module of the paged calls against torch's headers and libtkphi.so; returns its path.  What was
    built before does not outlive a build that fails: it may be of another interface."""
    import sysconfig

    import torch
    if os.path.exists(BINDING):
        os.remove(BINDING)
    root = _torch_root()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    # (-isystem: warnings of this module's own code only)
    include = [sysconfig.get_paths()["include"], os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wextra", "-DNDEBUG",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DTKPHI_TORCH_VERSION="{torch.__version__}"',
           "-o", BINDING, BINDING_SOURCE]
    for d in include:
        cmd += ["-isystem", d]
    cmd += [f"-L{os.path.dirname(LIB)}", "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN", f"-L{os.path.join(root, 'lib')}",
            f"-Wl,-rpath,{os.path.join(root, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("the C++ compiler failed building _paged_binding.so")
    if verbose or res.stderr:
        sys.stderr.write(res.stdout + res.stderr)
    return BINDING


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
