"""Builds liblvspec.so (sm_100a only) next to this file with nvcc, and _marshal.so, by which binding.py calls it, with gcc."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "liblvspec.so")
MARSHAL, MARSHAL_SRC = os.path.join(_HERE, "_marshal.so"), os.path.join(CSRC, "marshal.c")

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.h")) + \
        glob.glob(os.path.join(_ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_marshal(force: bool = False) -> None:
    """The calls' Python side; without Python's headers binding.py goes by ctypes."""
    include = sysconfig.get_paths()["include"]
    header = os.path.join(_ROOT, "include", "lvspec.h")
    if not os.path.exists(os.path.join(include, "Python.h")):
        return
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= max(map(os.path.getmtime, (MARSHAL_SRC, header))):
        return
    tmp = MARSHAL + f".{os.getpid()}.tmp"
    subprocess.run(["gcc", "-O2", "-fPIC", "-shared", "-Wall", "-Wextra", "-I", include, "-I", os.path.dirname(header),
                    "-o", tmp, MARSHAL_SRC], check=True)
    os.replace(tmp, MARSHAL)


def build(force: bool = False, verbose: bool = False) -> str:
    build_marshal(force)
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(_ROOT, "include"), "-I", CSRC]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    tmp = LIB + f".{os.getpid()}.tmp"
    cmd += ["-o", tmp, *sources()]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
