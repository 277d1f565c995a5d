"""Compile the CUDA sources into the in-tree shared library (sm_100a only)."""
from __future__ import annotations

import glob
import importlib.util
import os
import re
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libkeyformer_b200.so")
TORCH_SRC = os.path.join(CSRC, "kf_torch.cpp")      # torch side of the context-free operators, a CPython extension over the library
OBJ_DIR = os.path.join(ROOT, "_build")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _headers() -> list[str]:
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in sources() + _headers())


def _torch_dir() -> str:
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.submodule_search_locations:
        raise RuntimeError("torch is needed to build the extension")
    return list(spec.submodule_search_locations)[0]


def torch_lib() -> str:
    """Path of the extension for the installed torch and Python: one built for others is never loaded."""
    with open(os.path.join(_torch_dir(), "version.py")) as f:
        version = re.search(r"__version__ = '([^']+)'", f.read()).group(1)
    return os.path.join(PKG, f"_kf_torch.torch-{version}.{sysconfig.get_config_var('SOABI')}.so")


def build_torch(force: bool = False) -> str:
    """Build the extension that hands torch tensors to the library, if it is missing or older than its sources."""
    path = torch_lib()
    newest = max(os.path.getmtime(f) for f in (TORCH_SRC, os.path.join(ROOT, "include", "keyformer.h")))
    if not force and os.path.exists(path) and os.path.getmtime(path) >= newest:
        return path
    torch_dir = _torch_dir()
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    inc = [os.path.join(ROOT, "include"), os.path.join(torch_dir, "include"), os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
           os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    tmp = path + f".tmp{os.getpid()}"
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=1"] + [f"-I{d}" for d in inc] +
                          [TORCH_SRC, "-o", tmp, "-L" + PKG, "-l:" + os.path.basename(LIB), "-L" + os.path.join(torch_dir, "lib"), "-lc10", "-lc10_cuda",
                           "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libkeyformer_b200.so next to this file if it is missing or older than its sources, and the torch extension over it.
    Every .cu file is compiled to an object of its own (in parallel, only when it or a header changed)
    and the objects are linked into the library."""
    if not force and not _stale():
        build_torch()
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    hdr_time = max(os.path.getmtime(f) for f in _headers())
    common = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")
        if force or verbose or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(src), hdr_time):
            subprocess.check_call(common + ["-c", src, "-o", obj])
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sources()))
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.check_call([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-Xcompiler", "-fPIC", "-o", tmp] + objs)
    os.replace(tmp, LIB)
    build_torch(force)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
