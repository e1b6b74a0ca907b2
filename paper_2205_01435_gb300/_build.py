"""Builds in-tree: libwm.so (the C-ABI library, nvcc for sm_103a) and _seq_ext.so (the sequence
operators' Python marshalling, g++ against torch).  The library needs nothing of the module: where
that cannot be built (no torch or Python headers), a warning says why, and importing the sequence
operators' binding fails."""
from __future__ import annotations

import concurrent.futures as cf
import glob
import importlib.metadata
import os
import subprocess
import sysconfig
import warnings

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


def _headers():
    return glob.glob(os.path.join(INCLUDE, "*.h"))


def _fresh(product: str, deps: list[str]) -> bool:
    return os.path.exists(product) and all(os.path.getmtime(p) <= os.path.getmtime(product) for p in deps)


def _lib_fresh() -> bool:
    return _fresh(LIB, _sources() + _headers() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")))


def _ext_for() -> str:
    """What the marshalling module is built against: it holds the layouts of this torch and this Python."""
    try:
        torch = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        torch = "none"
    return f"torch {torch}, {sysconfig.get_config_var('SOABI')}\n"


def _ext_stamp() -> str:
    return os.path.join(BUILD, "wm_seq_ext.built_for")


def _ext_fresh() -> bool:
    if not _fresh(EXT, [EXT_SRC] + _headers()):
        return False
    try:
        with open(_ext_stamp()) as f:
            return f.read() == _ext_for()
    except OSError:
        return False


def up_to_date() -> bool:
    return _lib_fresh() and _ext_fresh()


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")
    return r.stdout + r.stderr


def _compile_ext():
    """The module's object, and the folder of torch's libraries."""
    import torch
    inc = os.path.join(os.path.dirname(torch.__file__), "include")
    nvcc = _nvcc()
    cuda = os.path.join(os.path.dirname(os.path.dirname(nvcc)) if os.path.isabs(nvcc) else "/usr/local/cuda", "include")
    obj = os.path.join(BUILD, "wm_seq_ext.o")
    _run(["g++", "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          "-I" + sysconfig.get_path("include"), "-I" + inc, "-I" + os.path.join(inc, "torch", "csrc", "api", "include"),
          "-I" + cuda, "-I" + INCLUDE, "-c", EXT_SRC, "-o", obj], "g++ on " + EXT_SRC)
    return obj, os.path.join(os.path.dirname(torch.__file__), "lib")


def _link_ext(obj, torch_lib):
    tmp = EXT + f".tmp{os.getpid()}"
    _run(["g++", "-shared", "-o", tmp, obj, "-L" + torch_lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda",
          "-L" + os.path.dirname(LIB), "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"], "link of " + EXT)
    os.replace(tmp, EXT)
    with open(_ext_stamp(), "w") as f:
        f.write(_ext_for())


def build(force: bool = False, verbose: bool = False, extra: list[str] | None = None) -> str:
    lib, ext = force or not _lib_fresh(), force or not _ext_fresh()
    if not lib and not ext:
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    nvcc = _nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        out = _run([nvcc, *ARCH, *NVCC_FLAGS, *(extra or []), "-c", src, "-o", obj], "nvcc on " + src)
        if verbose and out:
            print(out)
        return obj

    with cf.ThreadPoolExecutor(max_workers=max(1, min(8, os.cpu_count() or 1))) as ex:
        ext_obj = ex.submit(_compile_ext) if ext else None
        if lib:
            objs = list(ex.map(compile_one, _sources()))
            tmp = LIB + f".tmp{os.getpid()}"
            _run([nvcc, *ARCH, "-shared", "-o", tmp, *objs, "-lcudart", "-lcublas"], "link")
            os.replace(tmp, LIB)
    if ext:
        try:
            _link_ext(*ext_obj.result())
        except (RuntimeError, ImportError, OSError) as e:
            if os.path.exists(EXT):  # an older one, of other sources or another torch
                os.remove(EXT)
            warnings.warn(f"{os.path.basename(EXT)} was not built, so that the sequence operators' binding cannot be imported "
                          f"({os.path.basename(LIB)} is not affected): {e}", stacklevel=2)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
