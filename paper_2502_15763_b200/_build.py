"""Builds libhos.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
INCLUDE = os.path.join(_ROOT, "include")
LIB_PATH = os.path.join(_PKG, "libhos.so")
DEBUG_LIB_PATH = os.path.join(_PKG, "libhos_debug.so")   # the bounds-checked build (-DHOS_DEBUG_BOUNDS)

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "-t", "0"]


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + \
        glob.glob(os.path.join(INCLUDE, "*.h"))


def source_hash() -> str:
    """SHA-256 over the scheduling kernels' sources (names and contents, in name order), the headers that the
    KV-cache kernels share with them included: what a set of profiler counters of theirs was taken on.  Only
    the own files of the calls on the cache, on its pages and on drafts do not count."""
    import hashlib
    h = hashlib.sha256()
    for path in sorted(_deps()):
        if os.path.basename(path).startswith(("hos_kv", "hos_attn", "hos_pages", "hos_drafts", "hos_cluster")):
            continue
        h.update(os.path.basename(path).encode() + b"\0")
        with open(path, "rb") as fh:
            h.update(fh.read())
    return h.hexdigest()


def is_stale(debug: bool = False) -> bool:
    path = DEBUG_LIB_PATH if debug else LIB_PATH
    if not os.path.exists(path):
        return True
    t = os.path.getmtime(path)
    return any(os.path.getmtime(f) > t for f in _deps())


def build(force: bool = False, verbose: bool = False, debug: bool = False) -> str:
    """Compile every .cu under csrc/ into libhos.so (debug: the bounds-checked libhos_debug.so);
    returns its path."""
    path = DEBUG_LIB_PATH if debug else LIB_PATH
    if not force and not is_stale(debug):
        return path
    nvcc = os.environ.get("NVCC", "nvcc")
    tmp = path + f".{os.getpid()}.tmp"
    cmd = [nvcc] + NVCC_FLAGS + (["-DHOS_DEBUG_BOUNDS"] if debug else []) + (["-Xptxas", "-v"] if verbose else []) + \
        ["-I", INCLUDE, "-I", CSRC, "-o", tmp] + _sources()
    subprocess.check_call(cmd)
    os.replace(tmp, path)
    return path


# The Python module behind kv_cache.py: host code only, against the interpreter's and torch's headers.
BINDING_SOURCE = os.path.join(CSRC, "hos_kv_binding.cpp")


def binding_path() -> str:
    """Where the module for this interpreter and torch is: one built against other headers is never loaded."""
    import importlib.metadata
    import sysconfig
    return os.path.join(_PKG, f"_kv.torch-{importlib.metadata.version('torch')}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_binding(force: bool = False) -> str:
    """Compile hos_kv_binding.cpp into the module of binding_path(); returns that."""
    path = binding_path()
    newest = max(os.path.getmtime(f) for f in (BINDING_SOURCE, os.path.join(INCLUDE, "hos.h")))
    if not force and os.path.exists(path) and os.path.getmtime(path) >= newest:
        return path
    import sysconfig

    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(shutil.which(os.environ.get("NVCC", "nvcc")) or "/usr/local/cuda/bin/nvcc"))
    tmp = path + f".{os.getpid()}.tmp"
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", "-I", INCLUDE,
                           "-isystem", home + "/include", "-isystem", home + "/include/torch/csrc/api/include",
                           "-isystem", sysconfig.get_paths()["include"], "-isystem", cuda + "/include",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-o", tmp, BINDING_SOURCE,
                           "-L" + home + "/lib", "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"])
    os.replace(tmp, path)
    return path


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv, debug="--debug" in sys.argv))
    print(build_binding(force=True))
