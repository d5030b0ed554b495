"""Builds the CUDA library in-tree with nvcc for sm_100a (``libaccept.so`` beside this file).

Every source file is compiled by itself (objects under ``_build/``, side by side, only those whose own includes
have changed) and linked into the one library.

Besides the product there are two tests-only variants of the same sources (never loaded by the binding
unless a test asks for them):
  bounds  -DACCEPT_BOUNDS_CHECK: every access of a kernel to caller memory is checked against the byte
          ranges of the call, counted and skipped when outside (``libaccept_bounds.so``);
  stall   -DACCEPT_TEST_COPY_STALL: the staged batch-group encoder announces bytes that never arrive, so
          its bounded waits run out after 2 ms (``libaccept_stall.so``).
"""
from __future__ import annotations

import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJECTS = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libaccept.so")
SOURCES = [os.path.join(CSRC, f) for f in ("accept_api.cu", "accept_norm.cu", "accept_block.cu", "accept_matmul.cu")]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false",            # no FMA contraction: every fp32 operation rounds on its own
    "-Xcompiler", "-fPIC",
]

VARIANTS = {
    "bounds": (os.path.join(HERE, "libaccept_bounds.so"), ["-DACCEPT_BOUNDS_CHECK"]),
    "stall": (os.path.join(HERE, "libaccept_stall.so"), ["-DACCEPT_TEST_COPY_STALL"]),
}


def _includes(path: str, seen=None) -> set:
    """The file and every file of this repository that it includes."""
    seen = set() if seen is None else seen
    if path in seen:
        return seen
    seen.add(path)
    with open(path) as f:
        for name in re.findall(r'^#include "([^"]+)"', f.read(), re.M):
            _includes(os.path.normpath(os.path.join(os.path.dirname(path), name)), seen)
    return seen


def _older(target: str, files) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(f) > t for f in files)


def _stale(lib: str) -> bool:
    return any(_older(lib, _includes(s)) for s in SOURCES)


def needs_build() -> bool:
    return _stale(LIB)


def _nvcc() -> str:
    return os.environ.get("NVCC", "nvcc")


def _compile_jobs(lib: str, defines, force: bool, verbose: bool):
    """The commands that compile this library's stale objects."""
    os.makedirs(OBJECTS, exist_ok=True)
    jobs = []
    for source, obj in zip(SOURCES, _objects(lib)):
        if force or _older(obj, _includes(source)):
            jobs.append([_nvcc()] + NVCC_FLAGS + list(defines) + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, source])
    return jobs


def _objects(lib: str):
    name = os.path.splitext(os.path.basename(lib))[0]
    return [os.path.join(OBJECTS, name + "." + os.path.splitext(os.path.basename(s))[0] + ".o") for s in SOURCES]


def _run(commands) -> None:
    """Runs the commands side by side; raises if one fails."""
    jobs = [subprocess.Popen(c) for c in commands]
    failed = [j.args for j in jobs if j.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])


def _build(libs, force: bool, verbose: bool = False) -> None:
    """libs: (path, defines) of each library to bring up to date."""
    libs = [(lib, defines) for lib, defines in libs if force or _stale(lib)]
    _run([c for lib, defines in libs for c in _compile_jobs(lib, defines, force, verbose)])
    _run([[_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-o", lib] + _objects(lib) for lib, _ in libs])


def build(force: bool = False, verbose: bool = False) -> str:
    _build([(LIB, [])], force, verbose)
    return LIB


def build_variant(name: str, force: bool = False) -> str:
    """Builds (if stale) and returns the path of a tests-only variant."""
    _build([VARIANTS[name]], force)
    return VARIANTS[name][0]


def build_all(force: bool = False) -> None:
    """The product and the tests-only variants, compiled side by side."""
    _build([(LIB, [])] + list(VARIANTS.values()), force)


if __name__ == "__main__":
    import sys
    if "--all" in sys.argv:
        build_all(force="--force" in sys.argv)
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
