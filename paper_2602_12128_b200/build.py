"""Builds the CUDA library in-tree with nvcc for sm_100a (no GPU needed to compile)."""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libhla.so")
SOURCES = ["hla_api.cu", "hla_heads.cu", "hla_adamw.cu", "hla_scan.cu"]
OBJECTS = os.path.join(HERE, "_build")
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC",
]


def _newest_source_mtime() -> float:
    m = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(HERE), "include")):
        for f in os.listdir(root):
            m = max(m, os.path.getmtime(os.path.join(root, f)))
    return m


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _inputs(path: str, seen=None) -> set:
    """A source file and the headers of this project that it includes."""
    seen = set() if seen is None else seen
    if path not in seen:
        seen.add(path)
        with open(path) as f:
            for name in re.findall(r'^#include "([^"]+)"', f.read(), flags=re.M):
                _inputs(os.path.normpath(os.path.join(os.path.dirname(path), name)), seen)
    return seen


def _compile(source: str, force: bool, verbose: bool) -> str:
    path, obj = os.path.join(CSRC, source), os.path.join(OBJECTS, source + ".o")
    if not force and os.path.exists(obj) and os.path.getmtime(obj) >= max(os.path.getmtime(p) for p in _inputs(path) | {__file__}):
        return obj
    tmp = f"{obj}.{os.getpid()}"
    _run([nvcc_path()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", path, "-o", tmp], verbose)
    os.replace(tmp, obj)
    return obj


def _run(cmd, verbose):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles csrc/*.cu, one object each and side by side, and links libhla.so next to this file; returns its path."""
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    os.makedirs(OBJECTS, exist_ok=True)
    with ThreadPoolExecutor(len(SOURCES)) as pool:
        objects = list(pool.map(lambda s: _compile(s, force, verbose), SOURCES))
    tmp = f"{LIB}.{os.getpid()}"
    _run([nvcc_path()] + NVCC_FLAGS + ["-shared", "-lcuda"] + objects + ["-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
