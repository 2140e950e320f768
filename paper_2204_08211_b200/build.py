"""Builds libco3.so (CUDA kernels + C ABI) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
SOURCES = [os.path.join(_PKG, "csrc", f) for f in ("co3_kernels.cu", "co3_orth.cu", "co3_orth_small.cu", "co3_norm.cu", "co3_f8.cu", "co3_f8_linear.cu", "co3_f8_weight.cu", "co3_code_build.cc")]
HEADERS = [os.path.join(_PKG, "csrc", f) for f in ("co3_device.cuh", "co3_f8.cuh", "co3_launch.cuh", "co3_orth.cuh", "co3_orth_small.h", "co3_types.cuh")] + [os.path.join(_ROOT, "include", "co3.h")]
LIB = os.path.join(_PKG, "libco3.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-fmad=false",            # products and sums are written with explicit intrinsics; never contract
    "-Xcompiler", "-fPIC", "-shared", "--threads", "0",
]


def build(force: bool = False, verbose: bool = False) -> str:
    newest = max(os.path.getmtime(p) for p in SOURCES + HEADERS)
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= newest:
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = LIB + ".%d.tmp" % os.getpid()
    cmd = [nvcc, *NVCC_FLAGS, "-I", os.path.join(_ROOT, "include"), "-o", tmp, *SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
