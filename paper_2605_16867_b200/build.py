"""Builds libgoodserve.so (hand-written CUDA for sm_100a) in-tree with nvcc."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
INCLUDE = os.path.join(_ROOT, "include")
LIB_PATH = os.path.join(_PKG, "libgoodserve.so")
COUNT_LIB_PATH = os.path.join(_PKG, "libgoodserve_count.so")    # the measuring build (-DGS_COUNT_EVALS)
DEBUG_LIB_PATH = os.path.join(_PKG, "libgoodserve_debug.so")    # the checking build (-DGS_DEBUG)
SOURCES = ("api.cu", "prologue.cu", "route.cu", "risk.cu", "sequential.cu", "operators_api.cu", "experts_route.cu",
           "experts_linear.cu", "experts_combine.cu", "clip.cu")
MACRO_SOURCES = ("api.cu", "prologue.cu", "route.cu", "risk.cu", "sequential.cu")    # what -DGS_COUNT_EVALS and -DGS_DEBUG reach
OBJ_DIR = os.path.join(_PKG, "_build")
_compiled = set()                                               # objects that this process has built (and, while they are not stale, does not force again)
NVCC_FLAGS = ("-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-cudart", "shared")


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: libgoodserve.so cannot be built")


def _stale(path: str) -> bool:
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(INCLUDE, "goodserve.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False, extra_flags=(), counting: bool = False,
                  checking: bool = False) -> str:
    """Builds libgoodserve.so, or with ``counting`` the measuring build whose work counters tick,
    or with ``checking`` the build whose table index checks are compiled in."""
    path = COUNT_LIB_PATH if counting else DEBUG_LIB_PATH if checking else LIB_PATH
    if not force and not _stale(path):
        return path
    macros = ("-DGS_COUNT_EVALS",) if counting else ("-DGS_DEBUG",) if checking else ()
    # one compiler process per source file, side by side, then one link; the sources that neither of the
    # two macros reaches are compiled once for all three builds
    def compile_one(source: str) -> str:
        flags = (*NVCC_FLAGS, *extra_flags, *(macros if source in MACRO_SOURCES else ()))
        obj = os.path.join(OBJ_DIR, f"{hashlib.sha1(' '.join(flags).encode()).hexdigest()[:12]}_{source}.o")
        if not _stale(obj) and (obj in _compiled or not force):
            return obj
        cmd = [_nvcc(), *flags, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, source), "-o", f"{obj}.{os.getpid()}"]
        if verbose:
            print(" ".join(cmd), file=sys.stderr)
        subprocess.run(cmd, check=True)
        os.replace(f"{obj}.{os.getpid()}", obj)
        _compiled.add(obj)
        return obj
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=os.cpu_count() or 1) as workers:
        built = list(workers.map(compile_one, SOURCES))
    subprocess.run([_nvcc(), *NVCC_FLAGS, "--shared", *built, "-o", path + ".tmp"], check=True)
    os.replace(path + ".tmp", path)
    return path


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose=True,
                        extra_flags=("-Xptxas", "-v") if "--ptxas" in sys.argv else ()))
    if "--counting" in sys.argv:
        print(build_library(force="--force" in sys.argv, verbose=True, counting=True))
    if "--checking" in sys.argv:
        print(build_library(force="--force" in sys.argv, verbose=True, checking=True))
