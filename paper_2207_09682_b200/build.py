"""Builds libqgbdt.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _tensors.so, the module that
hands torch tensors to it, with the C++ compiler.

Every .cu file is compiled to an object of its own (in parallel, only when it or a header is
newer than the object), then the objects are linked into the shared library."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libqgbdt.so")
TENSORS_SRC = os.path.join(CSRC, "tensors.cpp")
TENSORS = os.path.join(HERE, "_tensors.so")
TENSORS_MADE_FOR = os.path.join(OBJ_DIR, "_tensors.txt")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-fmad=false",
    "-Xcompiler", "-fPIC",
]


def sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def headers() -> list[str]:
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _obj(src: str) -> str:
    return os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ".o")


def tensors_made_for() -> str:
    """What the extension module's binary interface depends on, besides its source."""
    import platform
    import sysconfig

    import torch
    return "torch %s, C++ ABI %d, Python %s %s\n" % (torch.__version__, torch._C._GLIBCXX_USE_CXX11_ABI, platform.python_version(),
                                                     sysconfig.get_config_var("SOABI"))


def tensors_stale() -> bool:
    try:
        with open(TENSORS_MADE_FOR) as f:
            if f.read() != tensors_made_for():
                return True
    except OSError:
        return True
    newest = max(os.path.getmtime(f) for f in [TENSORS_SRC, os.path.join(ROOT, "include", "qgbdt.h"), os.path.abspath(__file__)])
    return not os.path.exists(TENSORS) or os.path.getmtime(TENSORS) < newest


def build_tensors(force: bool = False) -> str:
    if not force and not tensors_stale():
        return TENSORS
    import sysconfig

    import torch
    torch_dir = os.path.dirname(torch.__file__)
    tmp = TENSORS + ".tmp.%d" % os.getpid()
    subprocess.check_call(
        [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
         "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(torch_dir, "include"),
         "-isystem", os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"],
         "-isystem", os.path.join(os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))), "include"),
         TENSORS_SRC, "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ltorch_cuda", "-o", tmp])
    os.replace(tmp, TENSORS)
    os.makedirs(OBJ_DIR, exist_ok=True)
    with open(TENSORS_MADE_FOR, "w") as f:
        f.write(tensors_made_for())
    return TENSORS


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in sources() + headers() + [os.path.abspath(__file__)])


def build(force: bool = False, verbose: bool = False) -> str:
    build_library(force, verbose)
    build_tensors(force)   # after the library, which does not need it
    return LIB


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    newest_header = max(os.path.getmtime(h) for h in headers() + [os.path.abspath(__file__)])

    def compile_one(src: str) -> str:
        obj = _obj(src)
        if (not force and os.path.exists(obj) and os.path.getmtime(obj) > os.path.getmtime(src)
                and os.path.getmtime(obj) > newest_header):
            return obj
        tmp = obj + ".tmp.%d" % os.getpid()
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + [
            "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", src, "-o", tmp]
        subprocess.check_call(cmd)
        os.replace(tmp, obj)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, sources()))
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([nvcc, "-shared", "-cudart", "static", "-gencode", "arch=compute_100a,code=sm_100a"]
                          + objs + ["-o", tmp])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
