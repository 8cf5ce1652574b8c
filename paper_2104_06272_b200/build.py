"""Builds libanakin.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _tokens_host.so (the Python module behind tokens.py) with g++.

Each .cu file is compiled to an object of its own (in parallel, only when it or a header changed) under
`_build/`, then the objects are linked into the shared library.  No relocatable device code is used: every
translation unit carries its own kernels.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libanakin.so")
HOST_SRC = os.path.join(CSRC, "tokens_host.cpp")
HOST = os.path.join(HERE, "_tokens_host.so")

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def headers():
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))


def _obj(src: str) -> str:
    return os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")


def _obj_stale(src: str, hdr_time: float) -> bool:
    o = _obj(src)
    return not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(src), hdr_time)


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in sources() + headers())


def host_stale() -> bool:
    header = os.path.join(ROOT, "include", "anakin.h")
    return not os.path.exists(HOST) or any(os.path.getmtime(p) > os.path.getmtime(HOST) for p in (HOST_SRC, header))


def build_host() -> None:
    """The module links to torch's libraries and to libanakin.so beside it."""
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    inc = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(torch, "include"),
           os.path.join(torch, "include", "torch", "csrc", "api", "include"), cuda]
    libs = ["-L", os.path.join(torch, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda", "-L", HERE, "-l:libanakin.so", "-Wl,-rpath,$ORIGIN"]
    tmp = HOST + f".tmp{os.getpid()}"
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared"] + [a for i in inc for a in ("-isystem", i)] + ["-o", tmp, HOST_SRC] + libs)
    os.replace(tmp, HOST)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or stale():
        build_lib(force, verbose)
    if force or host_stale():
        build_host()
    return LIB


def build_lib(force: bool, verbose: bool) -> None:
    os.makedirs(OBJ, exist_ok=True)
    hdr_time = max(os.path.getmtime(p) for p in headers())
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    todo = [s for s in sources() if force or _obj_stale(s, hdr_time)]

    def compile_one(src: str) -> None:
        tmp = _obj(src) + f".tmp{os.getpid()}"
        cmd = [NVCC] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + inc + ["-c", "-o", tmp, src]
        subprocess.check_call(cmd)
        os.replace(tmp, _obj(src))

    with ThreadPoolExecutor(max_workers=min(len(todo), os.cpu_count() or 4) or 1) as ex:
        list(ex.map(compile_one, todo))
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.check_call([NVCC, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", tmp] + [_obj(s) for s in sources()])
    os.replace(tmp, LIB)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
