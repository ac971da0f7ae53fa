"""Compile the CUDA library in-tree: paper_2407_19644_b200/libubp_b200.so (sm_100a).

    python -m paper_2407_19644_b200.build [--force] [--verbose] [--debug]

--debug builds libubp_b200_debug.so instead: the same library with -DUBP_DEBUG, in which the kernels that work on a plan
compare the indices they take from it or compute for shared / global memory with their extents, report a failure through the
plan's status word and skip the access (nothing traps). The row operators and those of the paged cache have no plan (the
attention kernels a status word of their own): they are the same in both builds. Load it by setting UBP_B200_LIBRARY to its path before the package is imported.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libubp_b200.so")
TORCH_SRC = os.path.join(CSRC, "python", "torch_calls.cpp")
TORCH_LIB = os.path.join(HERE, "_torch_calls.so")          # checks and allocations of the token-major calls, against torch
TORCH_MADE_FOR = os.path.join(HERE, "build", "torch_calls.txt")   # the torch and Python that it was built against
LIB_DEBUG = os.path.join(HERE, "libubp_b200_debug.so")     # the checked build (-DUBP_DEBUG): same entry points
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def _stale(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return True
    t = os.path.getmtime(lib)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.inc")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """The library, and where torch is installed the extension module of the token-major calls. The library comes first: it
    needs neither torch nor its headers."""
    lib = build_library(force, verbose, debug)
    if importlib.util.find_spec("torch") is not None:
        build_torch_calls(force)
    return lib


def build_library(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    lib = LIB_DEBUG if debug else LIB
    if not force and not _stale(lib):
        return lib
    objdir = os.path.join(HERE, "build_debug" if debug else "build")
    os.makedirs(objdir, exist_ok=True)
    common = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    common += os.environ.get("UBP_NVCC_FLAGS", "").split()      # extra flags, e.g. -DNAME for a diagnostic build
    if debug:
        common += ["-DUBP_DEBUG"]
    if verbose:
        common += ["-Xptxas", "-v"]
    objs = []
    procs = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src) + ".o")
        objs.append(obj)
        cmd = [NVCC, "-c", "-x", "cu" if src.endswith(".cu") else "c++", src, "-o", obj] + common
        procs.append((src, subprocess.Popen(cmd)))
    for src, p in procs:
        if p.wait() != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    tmp = lib + f".tmp{os.getpid()}"
    subprocess.run([NVCC, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"], check=True)
    os.replace(tmp, lib)
    return lib


def _torch_calls_stale(made_for: str) -> bool:
    deps = [TORCH_SRC, os.path.join(ROOT, "include", "ubp.h")]
    if not os.path.exists(TORCH_LIB) or any(os.path.getmtime(d) > os.path.getmtime(TORCH_LIB) for d in deps):
        return True
    try:
        with open(TORCH_MADE_FOR) as f:
            return f.read() != made_for
    except OSError:
        return True


def build_torch_calls(force: bool = False) -> str:
    """The extension module of the token-major calls (host code only; no CUDA source in it). It fits one torch and one Python:
    another version of either makes it stale."""
    import sysconfig
    import torch
    made_for = f"torch {torch.__version__}, {sysconfig.get_config_var('SOABI')}"
    if not force and not _torch_calls_stale(made_for):
        return TORCH_LIB
    base = os.path.dirname(torch.__file__)
    inc = [os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
           os.path.join(os.path.dirname(os.path.dirname(shutil.which(NVCC) or NVCC)), "include"), sysconfig.get_paths()["include"]]
    tmp = TORCH_LIB + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", TORCH_SRC, "-o", tmp,
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include")]
    for d in inc:
        cmd += ["-isystem", d]
    cmd += ["-L", os.path.join(base, "lib"), "-Wl,--no-as-needed", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"]
    subprocess.run(cmd, check=True)
    os.replace(tmp, TORCH_LIB)
    os.makedirs(os.path.dirname(TORCH_MADE_FOR), exist_ok=True)
    with open(TORCH_MADE_FOR, "w") as f:
        f.write(made_for)
    return TORCH_LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv, debug="--debug" in sys.argv))
