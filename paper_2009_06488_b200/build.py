"""Builds the CUDA library (csrc/*.cu -> libq4.so next to this file) for sm_100a, and the module that
hands torch tensors to it (csrc/q4_torch.cpp -> _q4_torch.so).

nvcc cross-compiles without a GPU.  The library links the CUDA runtime statically
and obtains the one driver entry point it needs at run time, so it loads on a
machine without a driver (its kernels obviously do not run there).
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libq4.so")
TORCH_SRC = os.path.join(CSRC, "q4_torch.cpp")
TORCH_LIB = os.path.join(HERE, "_q4_torch.so")      # tensors to the C ABI; links to libq4.so beside it

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-cudart", "static"]
OBJ_DIR = os.path.join(HERE, "_build")
TORCH_STAMP = os.path.join(OBJ_DIR, "q4_torch.built_for")      # torch and Python that the module was built for


def sources() -> list[str]:
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps() -> list[str]:
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    return sources() + hdrs + [os.path.join(INCLUDE, "q4.h")]


def _headers() -> list[str]:
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))] + \
           [os.path.join(INCLUDE, "q4.h")]


def build(force: bool = False, verbose: bool = False) -> str:
    """One object per source file (compiled in parallel, rebuilt when the source or any
    header is newer), then one link step."""
    from concurrent.futures import ThreadPoolExecutor
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    hdr_time = max(os.path.getmtime(h) for h in _headers())
    jobs, objs = [], []
    for src in sources():
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hdr_time):
            cmd = [nvcc, *NVCC_FLAGS, "-I", INCLUDE, "-I", CSRC, "-c", "-o", obj, src]
            if verbose:
                cmd[1:1] = ["-Xptxas", "-v"]
            jobs.append(cmd)
    if jobs:
        with ThreadPoolExecutor(max_workers=min(8, len(jobs))) as pool:
            for rc in pool.map(subprocess.call, jobs):
                if rc != 0:
                    raise subprocess.CalledProcessError(rc, "nvcc")
    if jobs or not os.path.exists(LIB):
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.check_call([nvcc, *NVCC_FLAGS, "-shared", "-o", tmp, *objs])
        os.replace(tmp, LIB)
    if force or not os.path.exists(TORCH_LIB) or _stamp() != _torch_and_python() or \
            os.path.getmtime(TORCH_LIB) < max(os.path.getmtime(TORCH_SRC), os.path.getmtime(os.path.join(INCLUDE, "q4.h"))):
        build_torch()
    return LIB


def _torch_and_python() -> str:
    import torch
    return f"{torch.__version__} {sys.implementation.cache_tag}"


def _stamp() -> str:
    try:
        with open(TORCH_STAMP) as f:
            return f.read()
    except OSError:
        return ""


def build_torch() -> None:
    """The marshalling module (host code only: g++ with torch's headers)."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    tmp = TORCH_LIB + f".tmp{os.getpid()}"
    subprocess.check_call(
        ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
         f'-DQ4_TORCH_VERSION="{torch.__version__}"',
         "-I", INCLUDE, "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
         "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
         "-isystem", os.environ.get("CUDA_HOME", "/usr/local/cuda") + "/include", "-o", tmp, TORCH_SRC,
         "-L", HERE, "-l:libq4.so", "-L", os.path.join(root, "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python",
         "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, TORCH_LIB)
    os.makedirs(OBJ_DIR, exist_ok=True)
    with open(TORCH_STAMP, "w") as f:
        f.write(_torch_and_python())


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
