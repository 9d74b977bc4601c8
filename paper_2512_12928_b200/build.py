"""Builds the CUDA library in-tree with nvcc for sm_100a, and the binding's module for torch tensors with g++.

    python -m paper_2512_12928_b200.build [--force] [--verbose]

Output: paper_2512_12928_b200/lib/libps_kvswap.so (C ABI declared in include/ps_kvswap.h) and beside it
_ps_tensor_args.<torch and Python>.so (where torch with CUDA is installed; the library does not need it).
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB_DIR = os.path.join(PKG, "lib")
LIB_PATH = os.path.join(LIB_DIR, "libps_kvswap.so")
SOURCES = ["ps_runtime.cu", "ps_swap.cu", "ps_step.cu", "ps_policy.cu", "ps_measure.cu", "ps_copy_kernels.cu",
           "ps_attn_kernels.cu", "ps_static_scratch.cu", "ps_slots.cu", "ps_rope.cu", "ps_paged_attn.cu"]
HEADERS = [os.path.join(CSRC, "ps_internal.h"), os.path.join(CSRC, "ps_ctx.h"), os.path.join(ROOT, "include", "ps_kvswap.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; set NVCC or put CUDA's bin directory on PATH")


TENSOR_ARGS_SOURCE = os.path.join(CSRC, "ps_tensor_args.cpp")


def tensor_args_path() -> str:
    """Where the module for torch tensors lies.  It is compiled against the insides of one torch and one Python, so its name
    has both: another torch finds no module rather than one that misreads its tensors."""
    import sysconfig

    import torch
    return os.path.join(LIB_DIR, f"_ps_tensor_args.torch-{torch.__version__}-abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}"
                                 f"{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_tensor_args(force: bool = False) -> str:
    """The module that takes torch tensors apart; nothing to do where torch is not installed or knows no CUDA."""
    import importlib.util
    if importlib.util.find_spec("torch") is None:
        return ""
    import sysconfig

    import torch
    if torch.version.cuda is None:
        return ""
    path = tensor_args_path()
    deps = [TENSOR_ARGS_SOURCE, os.path.join(ROOT, "include", "ps_kvswap.h")]
    if not force and os.path.exists(path) and all(os.path.getmtime(d) <= os.path.getmtime(path) for d in deps):
        return path
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    os.makedirs(LIB_DIR, exist_ok=True)
    partial = f"{path}.{os.getpid()}.tmp"     # another process may be loading the module meanwhile
    cmd = [shutil.which("g++") or "g++", "-shared", "-std=c++17", "-O2", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(base, "include"), "-I", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], "-I", os.path.join(cuda, "include"), "-o", partial,
           TENSOR_ARGS_SOURCE, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if proc.returncode != 0:
        if os.path.exists(partial):
            os.remove(partial)
        raise RuntimeError("g++ failed:\n" + proc.stdout[-4000:])
    os.replace(partial, path)
    return path


def needs_build() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB_PATH
    os.makedirs(LIB_DIR, exist_ok=True)
    cmd = [
        _nvcc(), "-shared", "-std=c++17", "-O3", "-lineinfo",
        "-gencode", "arch=compute_100a,code=sm_100a",
        "-Xcompiler", "-fPIC,-Wall,-Wno-unused-function",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC,
        "-o", LIB_PATH,
    ]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    proc = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if verbose or proc.returncode != 0:
        sys.stderr.write(proc.stdout)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout[-4000:])
    return LIB_PATH


def build(force: bool = False, verbose: bool = False) -> str:
    """The library first: it does not need the module."""
    build_library(force, verbose)
    build_tensor_args(force)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
