"""In-tree build of the CUDA library (``liblaga.so``) with nvcc for sm_100a, and of the compiled part of its Python binding
(``_binding.so``) with g++.

Run as ``python -m paper_2607_17644_b200.build`` or call :func:`build`.  nvcc cross-compiles
without a GPU present.  The library is rebuilt only when a source is newer than it, the binding also when torch or Python are others.
"""
from __future__ import annotations

import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
ROOT = os.path.dirname(PKG_DIR)
LIB_PATH = os.path.join(PKG_DIR, "liblaga.so")
BINDING_PATH = os.path.join(PKG_DIR, "_binding.so")
BINDING_STAMP = os.path.join(PKG_DIR, "_binding.built_with")     # the torch and the Python that _binding.so was built for
DEBUG_LIB_PATH = os.path.join(PKG_DIR, "liblaga_debug.so")   # the checked build (-DLAGA_DEBUG), see sm100_ptx.cuh

NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-shared", "--expt-relaxed-constexpr"]


def sources():
    return (sorted(glob.glob(os.path.join(CSRC, "*.cu"))),
            sorted(glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))))


def build_binding(force: bool = False, verbose: bool = False) -> str:
    """Build _binding.so (csrc/binding.cpp) against the headers of the installed torch.  With the system's g++ and not $CXX: torch's
    exceptions pass through it, so it must share torch's C++ runtime, which a compiler set up to link its own would not."""
    source, header = os.path.join(CSRC, "binding.cpp"), os.path.join(ROOT, "include", "laga.h")
    built_with = f"torch {importlib.metadata.version('torch')}\nPython {sys.version}\n"
    try:
        with open(BINDING_STAMP) as f:
            same = f.read() == built_with
    except OSError:
        same = False
    if (not force and same and os.path.exists(BINDING_PATH)
            and os.path.getmtime(BINDING_PATH) >= max(os.path.getmtime(source), os.path.getmtime(header))):
        return BINDING_PATH
    import torch
    base = os.path.dirname(torch.__file__)
    tmp = BINDING_PATH + f".tmp{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++20", "-fPIC", "-shared", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           *(f"-I{d}" for d in (os.path.join(base, "include"), os.path.join(base, "include", "torch", "csrc", "api", "include"),
                                sysconfig.get_paths()["include"], "/usr/local/cuda/include")),
           source, "-o", tmp, f"-L{os.path.join(base, 'lib')}", "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    subprocess.run(cmd, check=True)
    os.replace(tmp, BINDING_PATH)
    with open(tmp, "w") as f:
        f.write(built_with)
    os.replace(tmp, BINDING_STAMP)
    return BINDING_PATH


def build(force: bool = False, verbose: bool = False, extra_flags=(), debug: bool = False) -> str:
    """Build the library and then the binding (debug=True: the checked build, whose kernels verify their own index arithmetic
    and report LAGA_ERR_DEVICE_CHECK instead of making a bad access; selected at run time by LAGA_DEBUG=1).  The library needs neither
    g++ nor torch's headers, so a binding that cannot be built leaves it there."""
    path = build_library(force, verbose, extra_flags, debug)
    build_binding(force, verbose)
    return path


def build_library(force: bool = False, verbose: bool = False, extra_flags=(), debug: bool = False) -> str:
    cus, deps = sources()
    target = DEBUG_LIB_PATH if debug else LIB_PATH
    newest = max(os.path.getmtime(p) for p in cus + deps)
    if not force and os.path.exists(target) and os.path.getmtime(target) >= newest:
        return target
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = target + f".tmp{os.getpid()}"
    cmd = [nvcc, *NVCC_FLAGS, *(("-DLAGA_DEBUG=1",) if debug else ()), *extra_flags, "-o", tmp, *cus]
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    subprocess.run(cmd, check=True)
    os.replace(tmp, target)
    return target


if __name__ == "__main__":
    flags = ("-Xptxas", "-v") if "--ptxas-v" in sys.argv else ()
    print(build(force="--force" in sys.argv, verbose=True, extra_flags=flags))
    print(build(force="--force" in sys.argv, verbose=True, extra_flags=flags, debug=True))
