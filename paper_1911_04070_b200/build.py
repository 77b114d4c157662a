"""Compile the CUDA sources into paper_1911_04070_b200/libbpt.so for sm_100a, and the autograd functions over its C ABI
(csrc_torch/, C++ against PyTorch's headers) into paper_1911_04070_b200/_bpt_torch.so.

Usage: python -m paper_1911_04070_b200.build [--force] [--verbose]
nvcc cross-compiles without a GPU; the shared object stays inside the package
directory so that it travels with the source tree.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libbpt.so")
LIB_CHECK = os.path.join(HERE, "libbpt_check.so")   # the same sources with -DBPT_BOUNDS_CHECK (see csrc/bounds_check.cuh)
LIB_TORCH = os.path.join(HERE, "_bpt_torch.so")
SRC_TORCH = os.path.join(HERE, "csrc_torch", "autograd.cpp")
OBJ = os.path.join(HERE, "_build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _build_one(lib: str, tag: str, extra: list, force: bool, verbose: bool) -> str:
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    deps = srcs + glob.glob(os.path.join(CSRC, "*.cuh")) + [os.path.join(HERE, "..", "include", "bpt.h")]
    newest = max(os.path.getmtime(p) for p in deps)
    if not force and os.path.exists(lib) and os.path.getmtime(lib) >= newest:
        return lib
    os.makedirs(OBJ, exist_ok=True)
    procs, objs = [], []
    for s in srcs:
        o = os.path.join(OBJ, os.path.basename(s)[:-3] + tag + ".o")
        objs.append(o)
        if not force and os.path.exists(o) and os.path.getmtime(o) >= newest:
            continue
        cmd = [_nvcc()] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
        procs.append((cmd, subprocess.Popen(cmd)))
    for cmd, p in procs:
        if p.wait() != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    tmp = lib + ".tmp%d" % os.getpid()
    subprocess.check_call([_nvcc()] + NVCC_FLAGS[:2] + (["-rdc=true"] if "-rdc=true" in extra else []) + ["-shared", "-o", tmp] + objs + ["-lcudart"])
    os.replace(tmp, lib)
    return lib


_KEY_MARK = b"BPT_TORCH_KEY:"


def torch_key() -> str:
    """What _bpt_torch.so is compiled against: it fits this Python and this PyTorch only."""
    import torch
    return "torch %s, C++11 ABI %d, %s" % (torch.__version__, int(torch._C._GLIBCXX_USE_CXX11_ABI), sysconfig.get_config_var("SOABI"))


def built_for(path: str):
    """The torch_key a _bpt_torch.so was compiled with, read from the file without loading it; None if there is none."""
    try:
        with open(path, "rb") as f:
            data = f.read()
    except FileNotFoundError:
        return None
    at = data.find(_KEY_MARK)
    return None if at < 0 else data[at + len(_KEY_MARK):data.index(b"\0", at)].decode()


def _start_torch(force: bool):
    """Starts the compilation of _bpt_torch.so where it is out of date, or compiled for another PyTorch or Python; returns what
    _finish_torch takes."""
    deps = [SRC_TORCH, os.path.join(HERE, "..", "include", "bpt.h")]
    key = torch_key()
    if not force and built_for(LIB_TORCH) == key and os.path.getmtime(LIB_TORCH) >= max(os.path.getmtime(p) for p in deps):
        return None
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    inc = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include"),
           sysconfig.get_paths()["include"]]
    tmp = LIB_TORCH + ".tmp%d" % os.getpid()
    cmd = ["g++", "-O2", "-shared", "-fPIC", "-std=c++17", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           '-DBPT_TORCH_KEY="%s"' % key]
    cmd += [a for i in inc for a in ("-isystem", i)] + [SRC_TORCH, "-o", tmp, "-L" + os.path.join(root, "lib")]
    cmd += ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch", "-ltorch_python"]
    return cmd, subprocess.Popen(cmd), tmp


def _finish_torch(started):
    if started is None:
        return
    cmd, proc, tmp = started
    if proc.wait() != 0:
        raise RuntimeError("g++ failed: " + " ".join(cmd))
    os.replace(tmp, LIB_TORCH)


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds libbpt.so, the index-checking libbpt_check.so and _bpt_torch.so; returns the path of the first."""
    started = _start_torch(force)
    _build_one(LIB, "", [], force, verbose)
    # the checking build shares one violation record across its translation units: relocatable device code
    _build_one(LIB_CHECK, ".chk", ["-DBPT_BOUNDS_CHECK", "-rdc=true"], force, False)
    _finish_torch(started)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
