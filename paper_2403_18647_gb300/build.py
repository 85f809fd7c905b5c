"""Build libsdsat.so in-tree with nvcc for sm_103a (GB300).

Each .cu translation unit is compiled in parallel, then linked into one shared
library next to this file, beside the C part of the binding.  Used by __graft_entry__.build() and by the Python
binding's first use of either when it is missing or stale.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib
import os
import shlex
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
HEADER = os.path.join(ROOT, "include", "sdsat.h")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libsdsat.so")
# the part of the Python binding that is in C, for this interpreter alone (its name says which)
NATIVE = os.path.join(PKG, "_native" + sysconfig.get_config_var("EXT_SUFFIX"))
SOURCES = ["gemm.cu", "attention.cu", "accept.cu", "prefill.cu", "prefill_attention.cu", "pages.cu", "prefix_attention.cu",
           "logprobs.cu", "rotary.cu", "chunk_attention.cu", "adjust.cu", "sdsat.cu", "noalloc.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I" + os.path.join(ROOT, "include")]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _older(built: str, sources) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(f) > os.path.getmtime(built) for f in sources)


def is_stale() -> bool:
    """Whether the library has to be built."""
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".c")] + [HEADER, os.path.abspath(__file__)])


def native_is_stale() -> bool:
    """Whether the C part of the binding has to be built."""
    return _older(NATIVE, [os.path.join(CSRC, "binding.c"), HEADER, os.path.abspath(__file__)])


def build(verbose: bool = False, extra=()) -> str:
    """Both parts."""
    with cf.ThreadPoolExecutor(max_workers=1) as ex:
        native = ex.submit(build_native)
        lib = build_library(verbose, extra)
        native.result()
    return lib


def build_library(verbose: bool = False, extra=()) -> str:
    os.makedirs(BUILD, exist_ok=True)

    def one(src):
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        cmd = [nvcc(), *ARCH, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), r.stderr))
        if verbose and r.stderr.strip():
            print(r.stderr, file=sys.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [nvcc(), *ARCH, "-shared", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, LIB)
    return LIB


def cc():
    """The C compiler, as words: of the environment, else the one that built the interpreter, else the system's."""
    if os.environ.get("CC"):
        return shlex.split(os.environ["CC"])
    own = shlex.split(sysconfig.get_config_var("CC") or "")
    return own if own and shutil.which(own[0]) else ["cc"]


def build_native() -> str:
    tmp = NATIVE + ".tmp"
    include = sysconfig.get_paths()
    cmd = [*cc(), "-O2", "-shared", "-fPIC", "-fvisibility=hidden", "-I" + include["include"], "-I" + include["platinclude"],
           "-I" + os.path.join(ROOT, "include"), os.path.join(CSRC, "binding.c"), "-o", tmp]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError("no C compiler for the binding: %s" % e)
    if r.returncode != 0:
        raise RuntimeError("the C compiler failed:\n%s\n%s" % (" ".join(cmd), r.stderr))
    os.replace(tmp, NATIVE)
    importlib.invalidate_caches()   # (it is imported by the process that built it)
    return NATIVE


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
