"""Build ``libmxfp4.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU).

Each ``csrc/*.cu`` is compiled to an object of its own, all of them in parallel; an object is kept
in ``build/`` and compiled again only when its source or a header it includes has changed.

Run as ``python -m paper_2605_09825_b200.build`` or call :func:`build_library`.
"""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
OBJ_DIR = os.path.join(PKG_DIR, "build")
LIB_PATH = os.path.join(PKG_DIR, "libmxfp4.so")
BOUNDS_LIB_PATH = os.path.join(PKG_DIR, "libmxfp4_bounds.so")   # debug build, -DMXFP4_BOUNDS

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-std=c++17", "-lineinfo",
    "-Xcompiler", "-fPIC",
    "-Xptxas", "-v",
]


def _units():
    return [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith(".cu")]


def _depends(path: str, seen=None):
    """The source and every header it includes by a relative path, however deep."""
    seen = set() if seen is None else seen
    path = os.path.normpath(path)
    if path not in seen and os.path.exists(path):
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^\s*#include\s+"([^"]+)"', f.read(), flags=re.M):
                _depends(os.path.join(os.path.dirname(path), name), seen)
    return seen


def _stale(out: str, sources) -> bool:
    return not os.path.exists(out) or any(os.path.getmtime(s) > os.path.getmtime(out) for s in sources)


def needs_build(path: str = LIB_PATH) -> bool:
    return any(_stale(path, _depends(u)) for u in _units())


def _run(cmd, verbose: bool, what: str):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed building {what}")


def build_library(force: bool = False, verbose: bool = False, bounds: bool = False) -> str:
    """Build the library (``bounds=True``: the bounds-checking debug build, every computed
    shared-memory address checked, misses recorded in the status word instead of executed)."""
    path = BOUNDS_LIB_PATH if bounds else LIB_PATH
    if not force and not needs_build(path):
        return path
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    mine = f".tmp{os.getpid()}"

    def compile_unit(src):
        obj = os.path.join(OBJ_DIR, os.path.basename(src)[:-3] + ("_bounds.o" if bounds else ".o"))
        if force or _stale(obj, _depends(src)):
            flags = NVCC_FLAGS + (["-DMXFP4_BOUNDS"] if bounds else [])
            _run([nvcc] + flags + ["-c", "-o", obj + mine, src], verbose, os.path.basename(obj))
            os.replace(obj + mine, obj)
        return obj

    units = _units()
    with ThreadPoolExecutor(max_workers=len(units)) as pool:
        objs = list(pool.map(compile_unit, units))
    _run([nvcc] + NVCC_FLAGS[:2] + ["-shared", "-o", path + mine] + objs, verbose, os.path.basename(path))
    os.replace(path + mine, path)
    return path


if __name__ == "__main__":
    print(build_library(force=True, verbose=True, bounds="--bounds" in sys.argv))
