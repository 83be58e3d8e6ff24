"""Builds ``libspeca.so`` (CUDA kernels + C ABI) in-tree with nvcc for sm_100a.

Run as ``python -m paper_2509_11628_b200.build`` or call :func:`build`. nvcc cross-compiles
without a GPU, so the build also works on a CPU-only machine.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libspeca.so")
SOURCES = ["speca_kernels.cu", "speca_static.cu", "speca_layer_rows.cu", "speca_attention_bf16.cu", "speca_attention_f32.cu", "speca_attention_join.cu",
           "speca_norm8.cu", "speca_matmul8_tc.cu", "speca_matmul8_few.cu", "speca_matmul8_plan.cpp", "speca_api.cpp", "speca_layer.cpp", "speca_layer8.cpp"]
HEADERS = [os.path.join(CSRC, "speca_internal.h"), os.path.join(CSRC, "speca_layer_internal.h"),
           os.path.join(CSRC, "speca_layer_handle.h"), os.path.join(CSRC, "speca_rows_common.cuh"),
           os.path.join(CSRC, "speca_eight_common.cuh"), os.path.join(CSRC, "speca_tc.cuh"), os.path.join(CSRC, "speca_early.cuh"), os.path.join(CSRC, "speca_matmul8_common.cuh"), os.path.join(CSRC, "speca_matmul8_tensor.cuh"),
           os.path.join(CSRC, "speca_attention_common.cuh"), os.path.join(ROOT, "include", "speca.h")]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile if the library is missing or older than its sources; returns the library path."""
    if not force and not is_stale():
        return LIB
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [
        _nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--threads", "0",
        "-Xcompiler", "-fPIC,-O2,-Wall", "-shared", "-cudart", "static",
        "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", tmp,
    ] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError("nvcc failed:\n" + res.stdout)
    if verbose:
        print(res.stdout)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
