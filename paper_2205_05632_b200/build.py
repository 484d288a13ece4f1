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


# The operators' usual calls for torch: a Python extension beside the library, which it reaches through its addresses. It is built for one torch
# and one Python, whose versions stand beside it.
EXTENSION = os.path.join(HERE, "_torch_ops.so")
EXTENSION_SOURCE = os.path.join(CSRC, "torch_ops.cpp")


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


def _extension_stale(versions: str) -> bool:
    deps = [EXTENSION_SOURCE, os.path.join(HERE, "..", "include", "compams.h"), os.path.abspath(__file__)]
    if not os.path.exists(EXTENSION) or any(os.path.getmtime(p) > os.path.getmtime(EXTENSION) for p in deps):
        return True
    try:
        with open(EXTENSION + ".versions") as f:
            return f.read() != versions
    except OSError:
        return True


def build_extension(force: bool = False) -> None:
    import sysconfig

    try:
        import torch
    except ImportError:
        return  # the library is for programs without torch as well, the extension is not
    versions = "torch %s, Python %s" % (torch.__version__, sysconfig.get_config_var("SOABI"))
    if not force and not _extension_stale(versions):
        return
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.sep in _nvcc() else "/usr/local/cuda"
    tmp = EXTENSION + ".tmp.%d" % os.getpid()
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                    "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-isystem", os.path.join(root, "include"), "-isystem",
                    os.path.join(root, "include", "torch", "csrc", "api", "include"), "-isystem", os.path.join(cuda, "include"), "-isystem",
                    sysconfig.get_paths()["include"], EXTENSION_SOURCE, "-o", tmp, "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda",
                    "-ltorch_cpu", "-ltorch_python"], check=True)
    os.replace(tmp, EXTENSION)
    with open(EXTENSION + ".versions", "w") as f:
        f.write(versions)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = [_nvcc(), *NVCC_FLAGS, *(["-Xptxas", "-v"] if verbose else []),
               *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
        subprocess.run(cmd, check=True)
        os.replace(tmp, LIB)
    build_extension(force)  # (behind the library, which needs neither torch's headers nor a C++ compiler beside nvcc's)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
