"""Builds libgts.so in-tree with nvcc for sm_103a (GB300)."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
SRC = os.path.join(CSRC, "gts.cu")                  # the simulator (compiled through libgts.cu)
SOURCES = ("libgts.cu", "rotary.cu", "attention.cu", "prompt.cu", "pages.cu")
HDR = os.path.join(ROOT, "include", "gts.h")
BUILD_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD_DIR, "libgts.so")

NVCC_FLAGS = ["-gencode", "arch=compute_103a,code=sm_103a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC"]


def nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _inputs():
    """Every file libgts is made of."""
    include = os.path.join(ROOT, "include")
    return [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h"))] + [
        os.path.join(include, f) for f in os.listdir(include) if f.endswith(".h")]


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    newest = max(os.path.getmtime(f) for f in _inputs())
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= newest:
        return LIB
    tmp = LIB + f".{os.getpid()}.tmp"
    objects = [os.path.join(BUILD_DIR, f"{f[:-3]}.{os.getpid()}.o") for f in SOURCES]
    common = [nvcc()] + (["-Xptxas=-v"] if verbose else []) + NVCC_FLAGS + ["-I", os.path.join(ROOT, "include")]
    try:
        running = [subprocess.Popen(common + ["-c", "-o", o, os.path.join(CSRC, f)]) for f, o in zip(SOURCES, objects)]
        codes = [p.wait() for p in running]
        for p, rc in zip(running, codes):
            if rc:
                raise subprocess.CalledProcessError(rc, p.args)
        subprocess.check_call(common + ["-shared", "-o", tmp] + objects)
    finally:
        for o in objects:
            if os.path.exists(o):
                os.remove(o)
    os.replace(tmp, LIB)
    return LIB
