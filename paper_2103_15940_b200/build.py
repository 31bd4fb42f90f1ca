"""Builds the CUDA library in-tree: ``python -m paper_2103_15940_b200.build``.

``libqfmt.so``, next to this file, compiled by nvcc for sm_100a only, and ``_calls.abi3.so``, the part of the Python
binding that small passes need in C.
"""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqfmt.so")
CALLS = os.path.join(HERE, "_calls.abi3.so")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-ftz=false", "-prec-div=true", "-prec-sqrt=true", "-fmad=false",
    "-Xcompiler", "-fPIC", "-cudart", "static",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def needs_build() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(CALLS):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    deps = sources() + glob.glob(os.path.join(CSRC, "*.c")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    subprocess.check_call([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-fPIC", "-shared", "-I", sysconfig.get_paths()["include"],
                           "-I", os.path.join(ROOT, "include"), "-o", CALLS, os.path.join(CSRC, "calls.c")])
    # one nvcc per source, side by side; the objects are linked into the library and go
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources()]
        running = [subprocess.Popen([nvcc] + flags + ["-c", "-o", o, s]) for s, o in zip(sources(), objects)]
        codes = [p.wait() for p in running]
        for src, code in zip(sources(), codes):
            if code != 0:
                raise subprocess.CalledProcessError(code, f"{nvcc} -c {src}")
        subprocess.check_call([nvcc] + NVCC_FLAGS + ["-shared", "-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
