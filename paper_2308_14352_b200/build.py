"""Builds libemoe.so (the CUDA library) in-tree with nvcc for sm_100a, and _pycall (CPython callables of its entry points) for the
interpreter that runs this."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sysconfig
import warnings

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libemoe.so")
CALL_SOURCE = os.path.join(_HERE, "csrc", "pycall.cpp")
# an interpreter loads the file that carries its own tag, so that none gets another's
CALL_PATH = os.path.join(_HERE, "_pycall" + sysconfig.get_config_var("EXT_SUFFIX"))


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
        _build_calls()
    return LIB_PATH


def _build_calls() -> None:
    """The callables save the shortest calls a microsecond or two; where they cannot be built, ``binding`` makes those calls through ctypes."""
    include = sysconfig.get_paths()["include"]
    missing = [what for what, there in (("g++", shutil.which("g++")), ("Python.h", os.path.exists(os.path.join(include, "Python.h")))) if not there]
    if missing:
        warnings.warn(f"_pycall is not built ({' and '.join(missing)} not found): the training calls go through ctypes")
        return
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", include, "-o", CALL_PATH, CALL_SOURCE])


if __name__ == "__main__":
    print(build(force=True, verbose=True))
