"""Builds ``libmor_b200.so`` (the C-ABI library with the sm_100a kernels) in-tree with nvcc, and on top of it ``_ops.so`` (the
4-bit operators and the routing as torch operators: host code only) with g++.

Run as ``python -m paper_2512_22804_b200.build``.  nvcc cross-compiles, so no GPU is needed.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmor_b200.so")
SOURCES = ["mor_api.cu", "mor_kernels.cu", "mor_static.cu", "mor_main.cu", "mor_main_tensor.cu", "mor_main_row128.cu",
           "mor_main_blk128.cu", "mor_main_blk64.cu", "mor_main_col128.cu", "mor_main_channel.cu", "mor_main_dual.cu", "mor_main_colch.cu",
           "fp4/mor_fp4_quant.cu", "fp4/mor_fp4_gemm.cu", "fp4/mor_experts.cu"]
OBJ_DIR = os.path.join(HERE, "_build")
OPS_SOURCE = os.path.join(CSRC, "ops", "mor_ops.cpp")
OPS = os.path.join(HERE, "_ops.so")


def nvcc_path() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return p


def _deps():
    files = [os.path.join(d, f) for d, _, names in os.walk(CSRC) for f in names if f.endswith((".cu", ".cuh", ".h"))]
    return files + [os.path.join(ROOT, "include", "mor.h")]


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in _deps())


def build(force: bool = False, verbose: bool = False, lib: str = LIB, extra_flags=(), obj_dir=None) -> str:
    """Compile every source file to an object (side by side: the main kernel's instantiations are spread over
    several files for that purpose) and link the shared library."""
    if not force and lib == LIB and not needs_build():
        build_ops()
        return lib
    from concurrent.futures import ThreadPoolExecutor

    obj_dir = obj_dir or (OBJ_DIR if lib == LIB else lib + ".obj")
    os.makedirs(obj_dir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "--ftz=false", "--prec-div=true", "--prec-sqrt=true", "-Xfatbin", "-compress-all",
             "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    flags += list(extra_flags)
    if verbose:
        flags += ["-Xptxas", "-v"]
    newest = max(os.path.getmtime(d) for d in _deps() if d.endswith((".h", ".cuh")))

    def compile_one(src: str) -> str:
        obj = os.path.join(obj_dir, os.path.basename(src)[:-3] + ".o")
        path = os.path.join(CSRC, src)
        if force or verbose or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(path), newest):
            subprocess.run([nvcc_path(), *flags, "-c", path, "-o", obj], check=True)
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 4)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    subprocess.run([nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", *objs, "-o", lib], check=True)
    if lib == LIB:
        build_ops(force)
    return lib


def build_ops(force: bool = False) -> str:
    """Compile the torch operators against the installed torch; they find ``libmor_b200.so`` beside themselves."""
    header = os.path.join(ROOT, "include", "mor.h")
    if not force and os.path.exists(OPS) and os.path.getmtime(OPS) > max(os.path.getmtime(OPS_SOURCE), os.path.getmtime(header)):
        return OPS
    import sysconfig

    import torch

    t = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(nvcc_path()))
    include = [os.path.join(ROOT, "include"), os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    subprocess.run([shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-DTORCH_EXTENSION_NAME=_ops",
                    "-DTORCH_API_INCLUDE_EXTENSION_H", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *[f"-I{d}" for d in include], OPS_SOURCE, "-o", OPS, f"-L{os.path.join(t, 'lib')}", "-ltorch", "-ltorch_cpu", "-ltorch_python",
                    "-ltorch_cuda", "-lc10", "-lc10_cuda", f"-L{HERE}", "-l:libmor_b200.so", "-Wl,-rpath,$ORIGIN"], check=True)
    return OPS


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
