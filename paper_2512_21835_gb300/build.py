"""In-tree build of libloip.so for sm_103a (nvcc, one -gencode, TUs in parallel)."""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libloip.so")
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))  # the extension module of csrc/calls.c
BUILD = os.path.join(HERE, "_build")
SOURCES = ["decode.cu", "prefill.cu", "gemm_tc.cu", "attn_tc.cu", "pack.cu", "runtime.cu", "plan.cpp", "hostpool.cpp", "noalloc.cu",
           "disktier.cpp", "window.cu", "window_decode.cu", "window_prefill.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    for c in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libloip")


def _made() -> list:
    """What a build makes: the library, and the extension module where Python's headers are installed (without
    it the same entries are called through ctypes, a microsecond slower)."""
    return [OUT, CALLS] if os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")) else [OUT]


def _stale() -> bool:
    if not all(os.path.exists(f) for f in _made()):
        return True
    t = min(os.path.getmtime(f) for f in _made())
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "loip.h")]
    return any(os.path.getmtime(p) > t for p in deps if os.path.exists(p))


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return OUT
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)
    common = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-I", os.path.join(HERE, "..", "include")]

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
        cmd = [nvcc] + ARCH + common + ["-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and r.stderr:
            print(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    # Both files are made before either takes its place: an extension module never meets a library of other sources.
    lib, calls = os.path.join(BUILD, os.path.basename(OUT)), os.path.join(BUILD, os.path.basename(CALLS))

    def link(what, cmd):
        r = subprocess.run([nvcc] + cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {what}:\n{r.stdout}\n{r.stderr}")

    link("the library", ARCH + ["-shared", "-cudart", "shared", "-o", lib] + objs)
    if CALLS in _made():
        link("calls.c", ["-shared", "-cudart", "none", "-O2", "-Xcompiler", "-fPIC", "-I", sysconfig.get_paths()["include"],
                         os.path.join(CSRC, "calls.c"), "-o", calls, "-L", BUILD, "-lloip", "-Xlinker", "-rpath=$ORIGIN",
                         "-Xlinker", "--allow-shlib-undefined"])
    if os.path.exists(CALLS):
        os.remove(CALLS)
    os.replace(lib, OUT)
    if CALLS in _made():
        os.replace(calls, CALLS)
    return OUT


if __name__ == "__main__":
    print(build(force=True, verbose=True))
