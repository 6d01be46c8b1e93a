"""Builds the CUDA library in-tree (nvcc, sm_100a only). nvcc cross-compiles, so no GPU is needed to build."""
from __future__ import annotations

import glob
import os
import subprocess
import time
from concurrent.futures import ThreadPoolExecutor

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
LIB_PATH = os.path.join(_PKG, "libhashevict.so")
_SOURCES = sorted(glob.glob(os.path.join(_PKG, "csrc", "*.cu")))
_HEADERS = sorted(glob.glob(os.path.join(_ROOT, "include", "*.h")) + glob.glob(os.path.join(_PKG, "csrc", "*.cuh")) +
                  glob.glob(os.path.join(_PKG, "csrc", "*.h")))

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC",
]


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


DEBUG_LIB_PATH = os.path.join(_PKG, "libhashevict_debug.so")
_OBJ_DIR = os.path.join(_PKG, "build")


def _fresh(obj: str, deps: str, source: str) -> bool:
    """Whether an object was made from this source file (not from that of a tree that it was copied with) and nothing that it read is newer."""
    if not (os.path.exists(obj) and os.path.exists(deps)):
        return False
    with open(deps) as f:
        read = f.read().replace("\\\n", " ").partition(":")[2].split()
    return os.path.abspath(source) in map(os.path.abspath, read) and \
        all(os.path.exists(p) and os.path.getmtime(p) <= os.path.getmtime(obj) for p in read + [os.path.abspath(__file__)])


def _object(source: str, debug: bool, force: bool, verbose: bool) -> str:
    """One translation unit; compiled again when it or a header that it read the last time is newer than its object."""
    obj = os.path.join(_OBJ_DIR, os.path.basename(source)[:-3] + ("_debug.o" if debug else ".o"))
    deps = obj[:-2] + ".d"
    if not force and _fresh(obj, deps, source):
        return obj
    os.makedirs(_OBJ_DIR, exist_ok=True)
    tmp, began = f"{obj}.tmp{os.getpid()}", time.time()
    subprocess.run([nvcc_path()] + NVCC_FLAGS + (["-DHE_BOUNDS_CHECK"] if debug else []) + (["-Xptxas", "-v"] if verbose else []) +
                   ["-I", os.path.join(_ROOT, "include"), "-MD", "-MF", tmp + ".d", "-MT", "object", "-c", "-o", tmp, source], check=True)
    os.utime(tmp, (began, began))  # a source edited meanwhile is newer
    os.replace(tmp + ".d", deps)   # (both whole at any time: another process may be building too)
    os.replace(tmp, obj)
    return obj


def build_cuda(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compile csrc/*.cu into libhashevict.so, the translation units side by side; rebuilds only when a source or header is newer.

    debug=True builds libhashevict_debug.so with -DHE_BOUNDS_CHECK instead: every slot and token index is range-checked
    before it is used as an address, a failed check skips the access and raises he_device_error_count(). The binding
    loads that library when HE_DEBUG_LIB=1 is set before the first call."""
    out = DEBUG_LIB_PATH if debug else LIB_PATH
    deps = _SOURCES + _HEADERS
    if not force and os.path.exists(out) and all(os.path.getmtime(out) >= os.path.getmtime(p) for p in deps):
        return out
    began = time.time()
    with ThreadPoolExecutor(len(_SOURCES)) as pool:
        objects = list(pool.map(lambda s: _object(s, debug, force, verbose), _SOURCES))
    tmp = out + f".tmp{os.getpid()}"
    subprocess.run([nvcc_path()] + NVCC_FLAGS + ["-shared", "-o", tmp] + objects, check=True)
    os.utime(tmp, (began, began))
    os.replace(tmp, out)
    return out
