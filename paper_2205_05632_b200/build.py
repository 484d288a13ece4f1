"""Compile the CUDA library in-tree for sm_100a: `python -m paper_2205_05632_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcompams.so")
SOURCES = ["api.cu", "dense.cu", "blocksign.cu", "topk.cu", "randk.cu", "noalloc.cu", "collect.cu", "norm.cu", "adapter.cu", "head.cu", "clip.cu", "block.cu"]
HEADERS = ["common.cuh", "rows.cuh", "tcgen05.cuh", "adapter_tensor.cuh", "head_tensor.cuh", "context.h", "scatter.cuh", "select.cuh", "predict.cuh", os.path.join("..", "..", "include", "compams.h")]

# -fmad=false: no fused multiply-add anywhere, so each fp32 operation of the update rounds on its own.
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-fmad=false", "--threads", "0",
    "-Xcompiler", "-fPIC", "-shared",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS] + [os.path.abspath(__file__)]
    return any(os.path.getmtime(p) > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
           *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
