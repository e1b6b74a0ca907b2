"""Builds in-tree: libwm.so (the C-ABI library, nvcc for sm_103a) and _seq_ext.so (the sequence
operators' Python marshalling, g++ against torch)."""
from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libwm.so")
BUILD = os.path.join(PKG, "_build")
EXT = os.path.join(PKG, "_seq_ext.so")
EXT_SRC = os.path.join(CSRC, "wm_seq_ext.cpp")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I" + INCLUDE,
              "-Xptxas", "-warn-spills", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return (_sources() + [EXT_SRC] + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h"))
            + glob.glob(os.path.join(INCLUDE, "*.h")))


def up_to_date() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(EXT):
        return False
    t = min(os.path.getmtime(LIB), os.path.getmtime(EXT))
    return all(os.path.getmtime(p) <= t for p in _deps())


def build(force: bool = False, verbose: bool = False, extra: list[str] | None = None) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()
    extra = list(extra or [])

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        cmd = [nvcc, *ARCH, *NVCC_FLAGS, *extra, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout + r.stderr)
        return obj

    def run(cmd, what):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")

    def compile_ext():
        import torch
        inc = os.path.join(os.path.dirname(torch.__file__), "include")
        cuda = os.path.join(os.path.dirname(os.path.dirname(nvcc)) if os.path.isabs(nvcc) else "/usr/local/cuda", "include")
        obj = os.path.join(BUILD, "wm_seq_ext.o")
        run(["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
             "-I" + sysconfig.get_path("include"), "-I" + inc, "-I" + os.path.join(inc, "torch", "csrc", "api", "include"),
             "-I" + cuda, "-I" + INCLUDE, "-c", EXT_SRC, "-o", obj], "g++ on " + EXT_SRC)
        return obj, os.path.join(os.path.dirname(torch.__file__), "lib")

    with cf.ThreadPoolExecutor(max_workers=max(1, min(8, os.cpu_count() or 1))) as ex:
        ext = ex.submit(compile_ext)
        objs = list(ex.map(compile_one, _sources()))
        ext_obj, torch_lib = ext.result()
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-lcudart", "-lcublas"]
    run(cmd, "link")
    os.replace(tmp, LIB)
    tmp = EXT + f".tmp{os.getpid()}"
    run(["g++", "-shared", "-o", tmp, ext_obj, "-L" + torch_lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
         "-L" + PKG, "-l:libwm.so", "-Wl,-rpath,$ORIGIN"], "link of " + EXT)
    os.replace(tmp, EXT)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
