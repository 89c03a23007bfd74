"""Builds libsadmm.so in-tree from csrc/ with nvcc for sm_103a.

Each translation unit compiles in parallel; the objects link into one shared
library with the CUDA runtime linked statically, so the library loads
alongside any other CUDA user in the process.  No cmake: the C ABI in
include/sadmm.h is the library's only interface.  One host file beside it,
csrc/torch_ffn.cpp, is compiled against the torch of this interpreter: the
feed-forward functions' arguments and outputs as torch tensors.

The debug library (_build/debug/libsadmm.so, -DSADMM_DEBUG) adds index checks
to the kernels' global loads and stores: an index outside its buffer skips the
access and raises SADMM_EBOUNDS through sadmm_last_device_status.  The
binding loads it when the environment sets SADMM_DEBUG=1.
"""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys
from typing import List

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(BUILD, "libsadmm.so")
DEBUG_LIB = os.path.join(BUILD, "debug", "libsadmm.so")

SOURCES = ["abi.cu", "project.cu", "pack.cu", "conv_fwd.cu", "conv_slab.cu", "admm.cu", "elements.cu", "gemm.cu",
           "bwd.cu", "bwd_slab.cu", "bwd_grid.cu", "conv_grid.cu", "sparse.cu", "abi_ffn.cu", "norm.cu", "linear.cu",
           "tgemm.cu", "tgemm_pair.cu", "few.cu", "abi_q8.cu", "rms.cu", "quant.cu", "linear8.cu", "q8gemm.cu", "q8pair.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def nvcc() -> str:
    cand = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(cand):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return cand


def common_flags(extra: List[str]) -> List[str]:
    return ARCH + ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-O2",
                   "-I", INCLUDE, "-I", CSRC] + extra


def _inputs() -> List[str]:
    deps = [os.path.join(CSRC, s) for s in SOURCES]
    for fn in os.listdir(CSRC):
        if fn.endswith((".cuh", ".h")):
            deps.append(os.path.join(CSRC, fn))
    deps.append(os.path.join(INCLUDE, "sadmm.h"))
    return deps


def debug_requested() -> bool:
    return os.environ.get("SADMM_DEBUG", "") not in ("", "0")


def up_to_date(lib: str = LIB) -> bool:
    if not os.path.exists(lib):
        return False
    t = os.path.getmtime(lib)
    return all(os.path.getmtime(p) <= t for p in _inputs())


def build(force: bool = False, verbose: bool = False, extra: List[str] | None = None,
          debug: bool | None = None) -> str:
    """Compile csrc/*.cu and link _build/libsadmm.so (with debug, or SADMM_DEBUG=1
    in the environment: _build/debug/libsadmm.so with -DSADMM_DEBUG).  Returns
    the library path."""
    if debug is None:
        debug = debug_requested()
    lib = DEBUG_LIB if debug else LIB
    if not force and not extra and up_to_date(lib):
        return lib
    out = os.path.dirname(lib)
    os.makedirs(out, exist_ok=True)
    flags = common_flags(list(extra or []) + (["-DSADMM_DEBUG"] if debug else []))
    exe = nvcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(out, os.path.splitext(src)[0] + ".o")
        cmd = [exe] + flags + ["-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            sys.stderr.write(r.stdout + r.stderr)
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = lib + f".tmp{os.getpid()}"
    cmd = [exe] + ARCH + ["-shared", "-o", tmp] + objs + ["-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)
    return lib


TORCH_LIB = os.path.join(BUILD, "torch_ffn.so")


def build_torch_binding(force: bool = False) -> str:
    """Compile csrc/torch_ffn.cpp, the feed-forward operators' binding, against the
    torch of this interpreter (host code only).  Returns the module's path."""
    import sysconfig

    import torch
    src = os.path.join(CSRC, "torch_ffn.cpp")
    made_for = f"{sys.version} torch {torch.__version__}"
    note = TORCH_LIB + ".for"
    if not force and os.path.exists(TORCH_LIB) and os.path.exists(note) and open(note).read() == made_for:
        t = os.path.getmtime(TORCH_LIB)
        deps = [os.path.join(CSRC, h) for h in ("torch_call.h", "torch_q8.h")] + [os.path.join(INCLUDE, "sadmm.h")]
        if all(os.path.getmtime(p) <= t for p in [src] + deps):
            return TORCH_LIB
    os.makedirs(BUILD, exist_ok=True)
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    tmp = TORCH_LIB + f".tmp{os.getpid()}"
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={abi}", "-I", INCLUDE, "-I", CSRC,
           "-I", sysconfig.get_paths()["include"], "-isystem", os.path.join(base, "include"),
           "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", os.path.join(cuda, "include"), src, "-o", tmp, "-L", os.path.join(base, "lib"),
           "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on torch_ffn.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, TORCH_LIB)
    with open(note, "w") as f:
        f.write(made_for)
    return TORCH_LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True,
                extra=["-Xptxas", "-v"] if "--ptxas-v" in sys.argv else None))
