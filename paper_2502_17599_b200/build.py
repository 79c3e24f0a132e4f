"""Builds libmeda.so (the C-ABI CUDA library, nvcc for sm_100a) and _pages.so (the paged calls' argument
marshalling, g++ with torch's headers) in-tree."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libmeda.so")
BINDING_PATH = os.path.join(HERE, "_pages.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-lineinfo", "-std=c++17",
    "--shared", "-Xcompiler", "-fPIC",
    "-Xcompiler", "-fvisibility=hidden",
    "--expt-relaxed-constexpr",
]


def sources() -> list[str]:
    return [os.path.join(CSRC, "meda.cu")]


def _deps() -> list[str]:
    out = []
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for name in sorted(os.listdir(root)):
            if name.endswith((".cu", ".cuh", ".h")):
                out.append(os.path.join(root, name))
    return out


def is_stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    return any(os.path.getmtime(p) > t for p in _deps())


def binding_sources() -> list[str]:
    return [os.path.join(CSRC, "pages_binding.cpp")]


def binding_tag() -> bytes:
    """What _pages.so is built for: it uses torch's C++ classes and the interpreter's ABI, and holds this text."""
    import sysconfig

    import torch
    return f"built for torch {torch.__version__}, {sysconfig.get_config_var('SOABI')}".encode()


def binding_matches() -> bool:
    """Whether _pages.so is there and was built for this torch and interpreter."""
    if not os.path.exists(BINDING_PATH):
        return False
    with open(BINDING_PATH, "rb") as f:
        return binding_tag() + b"\0" in f.read()


def binding_is_stale() -> bool:
    if not binding_matches():
        return True
    t = os.path.getmtime(BINDING_PATH)
    header = os.path.join(os.path.dirname(HERE), "include", "meda.h")
    return any(os.path.getmtime(p) > t for p in binding_sources() + [header])


def _binding_command() -> list[str]:
    import sysconfig

    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"))
    cxx = shutil.which("g++")
    if cxx is None:
        raise RuntimeError("g++ not found: cannot build _pages.so")
    abi = f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}"
    return [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", abi, f'-DMEDA_BUILT_FOR="{binding_tag().decode()}"',
            "-I" + os.path.join(base, "include"), "-I" + os.path.join(base, "include", "torch", "csrc", "api", "include"),
            "-I" + os.path.join(cuda, "include"), "-I" + sysconfig.get_paths()["include"],
            *binding_sources(), "-o", BINDING_PATH, "-L" + os.path.join(base, "lib"), "-Wl,-rpath," + os.path.join(base, "lib"),
            "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def build_binding(force: bool = False) -> str:
    """Compiles _pages.so where it is missing, older than its sources or built for another torch; returns its path."""
    if force or binding_is_stale():
        res = subprocess.run(_binding_command(), capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("g++ failed:\n" + res.stdout + res.stderr)
    return BINDING_PATH


def build_library(force: bool = False, verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """Compiles libmeda.so where it is missing or older than its sources; returns its path.  Needs neither torch nor its headers."""
    if not force and not is_stale():
        return LIB_PATH
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        raise RuntimeError("nvcc not found: cannot build libmeda.so")
    cmd = [nvcc] + NVCC_FLAGS + (extra_flags or []) + ["-o", LIB_PATH] + sources()
    if verbose:
        print(" ".join(cmd), file=sys.stderr)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose and (res.stdout or res.stderr):
        print(res.stdout + res.stderr, file=sys.stderr)
    return LIB_PATH


def build(force: bool = False, verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """Compiles the library, then the paged calls' marshalling, where they are out of date; returns the library's path."""
    path = build_library(force, verbose, extra_flags)
    build_binding(force)
    return path


if __name__ == "__main__":
    flags = ["-Xptxas", "-v"] if "--ptxas" in sys.argv else None
    if importlib.util.find_spec("torch") is None:          # the C library alone, for callers that have no torch
        print("torch is not installed: _pages.so (the paged calls of binding.py) is not built", file=sys.stderr)
        build_library(force="--force" in sys.argv, verbose=True, extra_flags=flags)
    else:
        build(force="--force" in sys.argv, verbose=True, extra_flags=flags)
    print(LIB_PATH)
