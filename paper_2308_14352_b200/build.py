"""Builds libemoe.so (the CUDA library) in-tree with nvcc for sm_100a, and _pycall.so (CPython callables of its entry points)."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libemoe.so")
CALL_PATH, CALL_SOURCE = os.path.join(_HERE, "_pycall.so"), os.path.join(_HERE, "csrc", "pycall.cpp")


def sources():
    return sorted(glob.glob(os.path.join(_HERE, "csrc", "*.cu")))


def needs_build() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = sources() + glob.glob(os.path.join(_HERE, "csrc", "*.cuh")) + \
        glob.glob(os.path.join(_HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or needs_build():
        cmd = ["nvcc", "--threads", "0", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
               "-shared", "-Xcompiler", "-fPIC", "-o", LIB_PATH] + sources()
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        subprocess.check_call(cmd)
    if force or not os.path.exists(CALL_PATH) or os.path.getmtime(CALL_SOURCE) > os.path.getmtime(CALL_PATH):
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", sysconfig.get_paths()["include"], "-o", CALL_PATH, CALL_SOURCE])
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose=True))
