"""Compile the CUDA library in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(CSRC, "libmoe_route.so")
SOURCES = ["moe_route.cu", "permute_static.cu", "mx_rows.cu", "mx_product.cu", "expert_product.cu", "norm_rows.cu"]
HEADERS = ["device_utils.cuh", "route_kernels.cuh", "scatter_kernels.cuh", "combine_kernels.cuh", "ep_kernels.cuh",
           "backward_kernels.cuh", "mx_format.cuh", "mx_scatter.cuh", "mx_product.h", "expert_product.h",
           "mx8_format.cuh", "tcgen05.cuh", "redispatch_kernels.cuh",
           os.path.join("..", "..", "include", "moe_route.h")]


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
           "-Xcompiler", "-fPIC", "--threads", "0", "-shared", "-o", tmp]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose="-v" in sys.argv))
