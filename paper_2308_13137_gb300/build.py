"""Builds libomq.so in-tree: every csrc/*.cu compiled for sm_103a in parallel, then linked; and the
CPython module _bind.so of the serving calls (csrc/bind.cpp, host code against torch's headers).

Usage: python -m paper_2308_13137_gb300.build  (or build_lib() from Python).
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build", "omq")
LIB = os.path.join(PKG, "libomq.so")
BIND_SRC = os.path.join(CSRC, "bind.cpp")
BIND = os.path.join(PKG, "_bind.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-I", INCLUDE, "-I", CSRC]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", shutil.which("nvcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("nvcc not found")


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))] + \
           [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]


def _compile(src: str, extra) -> str:
    obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
    newest = max(os.path.getmtime(p) for p in [src] + _deps())
    if os.path.exists(obj) and os.path.getmtime(obj) >= newest:
        return obj
    cmd = [_nvcc()] + ARCH + FLAGS + list(extra) + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stderr}")
    return obj


def _run(cmd, what: str):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stderr}")


def _compile_bind() -> str:
    import torch
    obj = os.path.join(BUILD, "bind.o")
    if os.path.exists(obj) and os.path.getmtime(obj) >= max(
            os.path.getmtime(p) for p in [BIND_SRC] + [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]):
        return obj
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include")
    _run([shutil.which("g++") or "g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-I", INCLUDE, "-isystem", inc, "-isystem", os.path.join(inc, "torch", "csrc", "api", "include"), "-isystem", cuda,
          "-isystem", sysconfig.get_paths()["include"], "-c", BIND_SRC, "-o", obj], f"g++ on {BIND_SRC}")
    return obj


def _link_bind(obj: str):
    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    if os.path.exists(BIND) and os.path.getmtime(BIND) >= max(os.path.getmtime(obj), os.path.getmtime(LIB)):
        return
    _run([shutil.which("g++") or "g++", "-shared", "-o", BIND + ".tmp", obj, f"-L{PKG}", "-l:libomq.so", f"-L{lib}", "-lc10", "-lc10_cuda",
          "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{lib}"], "link of _bind.so")
    os.replace(BIND + ".tmp", BIND)


def build_lib(verbose: bool = False, extra=()) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = _sources()
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as ex:
        bind = ex.submit(_compile_bind)
        objs = list(ex.map(lambda s: _compile(s, extra), srcs))
        bind = bind.result()
    _link(objs, verbose)
    _link_bind(bind)
    return LIB


def _link(objs, verbose: bool) -> str:
    if os.path.exists(LIB) and os.path.getmtime(LIB) >= max(os.path.getmtime(o) for o in objs):
        return LIB
    tmp = LIB + ".tmp"
    cmd = [_nvcc()] + ARCH + ["-shared", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build_lib(verbose=True, extra=sys.argv[1:])
