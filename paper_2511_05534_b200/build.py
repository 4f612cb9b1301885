"""Builds the CUDA library (libflowmm.so, nvcc for sm_100a) and the Python marshalling module beside it (_marshal.<tag>.so, g++) in-tree."""
from __future__ import annotations

import os
import re
import shutil
import subprocess
import sys
import sysconfig

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libflowmm.so")
DEBUG_LIB_PATH = os.path.join(_PKG, "libflowmm_debug.so")     # the same sources with -DFLOWMM_DEBUG (index checks)
SOURCES = ["flowmm_api.cu"]
MARSHAL_SOURCE = "marshal.cpp"


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != MARSHAL_SOURCE] + [os.path.join(_ROOT, "include", "flowmm.h")]
    return max(os.path.getmtime(p) for p in paths)


def nvcc_command(out: str, verbose_ptxas: bool = False, debug: bool = False):
    cmd = ["nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "-shared", "-cudart", "static", "-I", os.path.join(_ROOT, "include"), "-I", CSRC,
           "-o", out]
    if verbose_ptxas:
        cmd += ["-Xptxas", "-v"]
    if debug:
        cmd += ["-DFLOWMM_DEBUG"]
    return cmd + [os.path.join(CSRC, s) for s in SOURCES]


def marshal_path() -> str:
    """Where the marshalling module is that was built for this interpreter and this torch, whose objects' layouts it holds."""
    import torch
    tag = "%s.torch-%s" % (sysconfig.get_config_var("SOABI"), torch.__version__)
    return os.path.join(_PKG, "_marshal.%s.so" % re.sub(r"[^0-9A-Za-z.]+", "-", tag))


def _build_marshal(force: bool) -> None:
    path, source = marshal_path(), os.path.join(CSRC, MARSHAL_SOURCE)
    newest = max(os.path.getmtime(source), os.path.getmtime(os.path.join(_ROOT, "include", "flowmm.h")))
    if not force and os.path.exists(path) and os.path.getmtime(path) >= newest:
        return
    import torch
    from torch.utils import cpp_extension
    tmp = path + ".%d.tmp" % os.getpid()
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"))), "include")
    include = cpp_extension.include_paths() + [cuda, sysconfig.get_paths()["include"], os.path.join(_ROOT, "include")]
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
                           *("-I" + d for d in include), source, "-o", tmp,
                           *("-L" + d for d in cpp_extension.library_paths()), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    os.replace(tmp, path)


def build(force: bool = False, verbose_ptxas: bool = False, debug: bool = False) -> str:
    """Compile if the library is missing or older than any source; returns its path.  debug: the build with
    index checks (libflowmm_debug.so) instead of the release library."""
    path = DEBUG_LIB_PATH if debug else LIB_PATH
    if force or not os.path.exists(path) or os.path.getmtime(path) < _newest_source_mtime():
        tmp = path + ".%d.tmp" % os.getpid()
        subprocess.check_call(nvcc_command(tmp, verbose_ptxas, debug))
        os.replace(tmp, path)
    if not debug:
        _build_marshal(force)                # (last: the library needs neither g++ nor the headers of Python and torch)
    return path


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose_ptxas="-v" in sys.argv, debug="--debug" in sys.argv))
