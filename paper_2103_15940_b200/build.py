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


def headers():
    return glob.glob(os.path.join(ROOT, "include", "*.h"))


def older(target, deps) -> bool:
    """Whether a target is missing or older than what it is made of."""
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def library_needs_build() -> bool:
    return older(LIB, sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + headers())


def calls_need_build() -> bool:
    return older(CALLS, glob.glob(os.path.join(CSRC, "*.c")) + headers())


def needs_build() -> bool:
    return library_needs_build() or calls_need_build()


def build_library(verbose: bool = False) -> None:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    # one nvcc per source, side by side; the objects are linked into the library and go
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources()]
        running = [subprocess.Popen([nvcc] + flags + ["-c", "-o", o, s]) for s, o in zip(sources(), objects)]
        codes = [p.wait() for p in running]
        for src, code in zip(sources(), codes):
            if code != 0:
                raise subprocess.CalledProcessError(code, f"{nvcc} -c {src}")
        subprocess.check_call([nvcc] + NVCC_FLAGS + ["-shared", "-o", LIB] + objects)


def build_calls() -> None:
    subprocess.check_call([os.environ.get("CC", "gcc"), "-O2", "-Wall", "-fPIC", "-shared", "-I", sysconfig.get_paths()["include"],
                           "-I", os.path.join(ROOT, "include"), "-o", CALLS, os.path.join(CSRC, "calls.c")])


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds what is missing or out of date: the library first, since all calls but the sub-layer ones do without the module
    (which needs the interpreter's headers)."""
    if force or library_needs_build():
        build_library(verbose)
    if force or calls_need_build():
        build_calls()
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
