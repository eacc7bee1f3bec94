"""Builds libadapt_b200.so (CUDA kernels + C ABI) for sm_100a with nvcc, and _adapt_torch.so (the calls of the
training-step operators from torch tensors, g++), in-tree.

    python -m paper_2107_13490_b200.build [--force] [--check] [--library]

Without torch, or with --library, the library alone is built.  --check also builds libadapt_b200_check.so, the same library with every data-dependent table
index tested against its table's size (-DADAPT_CHECK_BOUNDS; see adapt_bounds_check_status).
"""
from __future__ import annotations

import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libadapt_b200.so")
CHECK_LIB = os.path.join(HERE, "libadapt_b200_check.so")
CALLS = os.path.join(HERE, "_adapt_torch.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    # no FMA contraction anywhere: every fp32 step that decides an integer is one IEEE operation
    "-fmad=false",
    "-shared", "-Xcompiler", "-fPIC", "-Xcompiler", "-ffp-contract=off",
    "-t", "0",      # the .cu files side by side, as many as there are cores
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + \
        [os.path.join(os.path.dirname(HERE), "include", "adapt.h")]


def build(force: bool = False, verbose: bool = False, check: bool = False, calls: bool = True) -> str:
    """Builds the library (or, with check=True, its bounds-checking twin) if it is stale, and the extension
    likewise where there is a torch to build it for, unless calls=False."""
    lib = CHECK_LIB if check else LIB
    stale = (not os.path.exists(lib)) or any(
        os.path.getmtime(d) > os.path.getmtime(lib) for d in _deps())
    if force or stale:
        nvcc = os.environ.get("NVCC", "nvcc")
        tmp = lib + ".tmp%d" % os.getpid()
        cmd = [nvcc] + NVCC_FLAGS + (["-DADAPT_CHECK_BOUNDS"] if check else []) + \
            (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + sources()
        subprocess.run(cmd, check=True)
        os.replace(tmp, lib)
    if calls and torch_version() is not None:
        build_calls(force)
    return lib


def torch_version() -> str | None:
    """The installed torch and the interpreter, what the extension is built for; None without a torch."""
    try:
        return "torch %s, python %s\n" % (importlib.metadata.version("torch"), sys.version.split()[0])
    except importlib.metadata.PackageNotFoundError:
        return None


def build_calls(force: bool = False) -> str:
    """Builds the extension behind binding.py's training-step operators if its source, torch or the interpreter
    changed."""
    source, header = os.path.join(CSRC, "torch_calls.cpp"), os.path.join(os.path.dirname(HERE), "include", "adapt.h")
    built_for, now = CALLS + ".built_for", torch_version()
    stale = (not os.path.exists(CALLS)) or any(
        os.path.getmtime(d) > os.path.getmtime(CALLS) for d in (source, header))
    if not stale:
        try:
            with open(built_for) as f:
                stale = f.read() != now
        except OSError:
            stale = True
    if force or stale:
        import torch
        root = os.path.dirname(torch.__file__)
        cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
        tmp = CALLS + ".tmp%d" % os.getpid()
        cmd = ["g++", "-O2", "-std=c++20", "-fPIC", "-shared", "-Wall"]
        cmd += ["-I" + d for d in (os.path.join(root, "include"), os.path.join(root, "include/torch/csrc/api/include"),
                                   sysconfig.get_paths()["include"], os.path.join(cuda, "include"))]
        cmd += [source, "-o", tmp, "-L" + os.path.join(root, "lib")]
        cmd += ["-l" + n for n in ("torch_python", "torch", "torch_cpu", "torch_cuda", "c10", "c10_cuda")]
        subprocess.run(cmd, check=True)
        os.replace(tmp, CALLS)
        with open(built_for, "w") as f:
            f.write(now)
    return CALLS


if __name__ == "__main__":
    how = dict(force="--force" in sys.argv, verbose="-v" in sys.argv, calls="--library" not in sys.argv)
    print(build(**how))
    if "--check" in sys.argv:
        print(build(**how, check=True))
