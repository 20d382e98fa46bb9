"""Builds the CUDA library in-tree for sm_100a with nvcc (no JIT cache involved)."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libskipdecode.so")
SOURCES = [os.path.join(CSRC, "skipdecode.cu")]
HEADERS = [os.path.join(CSRC, n) for n in ("kernels.cuh", "gemm_tc.cuh", "sample.cuh", "attn_prefill.cuh", "gemm_persist.cuh", "attn_stream.cuh",
                                              "paged.cuh", "attn_paged.cuh", "attn_chunk.cuh", "sample_rows.cuh", "cache_host.cuh")] + \
          [os.path.join(os.path.dirname(PKG), "include", "skipdecode.h")]


def nvcc_path() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    cmd = [nvcc_path(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC,-O2", "-shared", "-o", LIB] + SOURCES
    if verbose:
        cmd[1:1] = ["-Xptxas", "-v"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + res.stdout + res.stderr)
    if verbose:
        print(res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
