"""Compile the CUDA sources into libmtad.so (sm_100a only) next to this file, and the tensor form of its operators into _ops.so.

    python -m paper_2407_09722_b200.build [--verbose]
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmtad.so")
OPS = os.path.join(HERE, "_ops.so")
OPS_SRC = os.path.join(CSRC, "ops_py.cpp")
HEADER = os.path.join(ROOT, "include", "mtad.h")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _stale(target: str, deps) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _nvcc() -> str:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    return shutil.which(nvcc) or nvcc


def ops_stale() -> bool:
    """Whether _ops.so is older than its sources, or was built against another torch (whose name is in it)."""
    import torch
    if _stale(OPS, [OPS_SRC, HEADER]):
        return True
    with open(OPS, "rb") as f:
        return f"torch {torch.__version__};".encode() not in f.read()


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER]):
        cmd = [_nvcc(), "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-t", "0",
               "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
               "-o", LIB] + os.environ.get("MTAD_NVCC_FLAGS", "").split() + sources()
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)
    if force or ops_stale():
        build_ops(verbose)
    return LIB


def build_ops(verbose: bool = False) -> str:
    import torch
    t = os.path.dirname(os.path.abspath(torch.__file__))
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DMTAD_TORCH="torch {torch.__version__};"']
    for d in (os.path.join(ROOT, "include"), os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
              sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")):
        cmd += ["-I", d]
    # (libstdc++ by name, ahead of the compiler's own: one that comes with the archive only would put a second copy of it into the module, and
    # a number written to a stream of torch's then ends the process)
    cmd += [OPS_SRC, "-o", OPS, "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
            "-L", HERE, "-l:libmtad.so", "-l:libstdc++.so.6", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    return OPS


if __name__ == "__main__":
    build(force=True, verbose="--verbose" in sys.argv)
    print(LIB)
