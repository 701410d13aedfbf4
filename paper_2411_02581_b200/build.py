"""Builds the CUDA library for sm_100a with nvcc, in-tree (``_lib/libtuna.so``)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB_DIR = os.path.join(_HERE, "_lib")
LIB_PATH = os.path.join(LIB_DIR, "libtuna.so")
TORCH_PATH = os.path.join(LIB_DIR, "tuna_torch.so")   # the operator calls' torch marshalling (tuna_torch.cpp)
TORCH_SOURCE = os.path.join(CSRC, "tuna_torch.cpp")
SOURCES = ["tuna_plan.cu", "tuna_api.cu", "tuna_static.cu", "tuna_shard.cu", "tuna_move.cu",
           "tuna_route.cu", "tuna_balance.cu", "tuna_fp8.cu", "tuna_fp4.cu", "tuna_moe.cu", "tuna_few.cu"]
HEADERS = [os.path.join(CSRC, h) for h in ("tuna_internal.h", "tuna_plan.h", "tuna_plan_kernels.cuh", "tuna_ops.cuh", "tuna_fp8.h", "tuna_fp4.h", "tuna_route.cuh")] + [
    os.path.join(ROOT, "include", "tuna.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_made_for() -> str:
    """What a build of the marshalling fits: one torch and one Python."""
    import torch
    return f"torch {torch.__version__}, Python {sys.version_info.major}.{sys.version_info.minor}"


def build_torch(force: bool = False) -> str:
    """Compile the torch marshalling of the operator calls (host code only) for the torch and the Python that run."""
    deps = [TORCH_SOURCE, os.path.join(ROOT, "include", "tuna.h")]
    note, made_for = TORCH_PATH + ".made_for", _torch_made_for()
    if not force and os.path.exists(TORCH_PATH) and all(os.path.getmtime(d) <= os.path.getmtime(TORCH_PATH) for d in deps):
        if os.path.exists(note) and open(note).read() == made_for:
            return TORCH_PATH
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    os.makedirs(LIB_DIR, exist_ok=True)
    tmp = TORCH_PATH + ".tmp.%d" % os.getpid()
    try:
        subprocess.check_call(
            ["g++", "-O2", "-std=c++20", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
             "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(base, "include"),
             "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
             "-isystem", sysconfig.get_paths()["include"], "-isystem", "/usr/local/cuda/include", TORCH_SOURCE, "-o", tmp,
             "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10", "-ldl"])
    except (OSError, subprocess.CalledProcessError):
        if os.path.exists(TORCH_PATH):
            os.remove(TORCH_PATH)  # no old one is left for a load that would rather say that it is missing
        raise
    os.replace(tmp, TORCH_PATH)
    with open(note, "w") as f:
        f.write(made_for)
    return TORCH_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu file for sm_100a and link the shared library; then the torch marshalling, which the library
    does without: where torch is missing it is left out, and a failure is a warning (``moe`` says that it is missing)."""
    if force or needs_build():
        _build_library(verbose)
    if importlib.util.find_spec("torch") is not None:
        try:
            build_torch(force)
        except (OSError, subprocess.CalledProcessError) as e:
            warnings.warn(f"the torch marshalling of the operators was not built: {e}", RuntimeWarning)
    return LIB_PATH


def _build_library(verbose: bool) -> None:
    os.makedirs(LIB_DIR, exist_ok=True)
    tmp = LIB_PATH + ".tmp.%d" % os.getpid()
    cmd = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3",
           "-std=c++20", "-Xcompiler", "-fPIC", "--threads", "0", "-shared", "-cudart", "static",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES] + ["-o", tmp]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB_PATH)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
