"""Builds libkurtail.so (sm_100a, nvcc) and _serving.so (the Python side of its serving calls, g++) in-tree."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkurtail.so")
SERVING = os.path.join(HERE, "_serving.so")
SOURCES = ["kt_api.cu", "serve.cu"]
HEADERS = ["sm100_prims.cuh", "gemm_sm100.cuh", "elementwise.cuh", "fused_small.cuh", "small_orth.cuh", "serve.h",
           "serve_norm.cuh", "serve_cache.cuh", "serve_attend.cuh", "serve_prompt.cuh"]


def _nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _older(out, sources):
    """out is missing or older than one of its sources (or the header)."""
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    deps = [os.path.join(CSRC, f) for f in sources]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "kurtail.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def built_for():
    """The Python and the torch that _serving.so is built against; a module that names others is not used."""
    import torch
    return f"Python {sys.version.split()[0]}, torch {torch.__version__}"


def _serving_stale():
    """_serving.so is missing, older than its sources, or built against another Python or torch."""
    if _older(SERVING, ["binding.cpp"]):
        return True
    with open(SERVING, "rb") as f:
        return built_for().encode() + b"\0" not in f.read()


def needs_build():
    return _older(LIB, SOURCES + HEADERS) or _serving_stale()


def _run(cmd, verbose):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)


def build(force=False, verbose=False):
    """Compiles what is missing or older than its sources."""
    if force or _older(LIB, SOURCES + HEADERS):
        _run([_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-t", str(len(SOURCES)), "-shared", "-Xcompiler", "-fPIC", "-Xptxas", "-v" if verbose else "-warn-spills",
              "-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES], verbose)
    if force or _serving_stale():
        import torch
        root = os.path.dirname(torch.__file__)
        _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall",
              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DKT_BUILT_FOR="{built_for()}"',
              "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include"),
              "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
              "-o", SERVING, os.path.join(CSRC, "binding.cpp"), "-L" + os.path.join(root, "lib"),
              "-lc10", "-ltorch_cpu", "-ltorch_python"], verbose)
    return LIB


if __name__ == "__main__":
    import sys
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
