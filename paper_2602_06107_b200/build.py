"""Builds libjackpot.so (sm_100a only) in-tree with nvcc."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libjackpot.so")
SOURCES = ["jp_api.cu", "jp_stream.cu", "jp_epilogue.cu", "jp_grad.cu", "jp_noalloc.cu", "jp_probe.cu", "jp_rowlambda.cu", "jp_vshard.cu", "jp_sparse.cu", "jp_lmhead.cu", "jp_norm.cu", "jp_w4.cu", "jp_verify.cu", "jp_loss.cu", "jp_block.cu", "jp_i8.cu"]
HEADERS = ["jp_common.cuh", "jp_internal.h", "jp_pairs.cuh"]


def _newest_source() -> float:
    paths = [os.path.join(CSRC, f) for f in SOURCES + HEADERS] + [os.path.join(ROOT, "include", "jackpot.h")]
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-shared", "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB] + [os.path.join(CSRC, f) for f in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
