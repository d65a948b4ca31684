"""Builds the CUDA shared library in-tree with nvcc for sm_100a.

    python -m paper_2505_01637_b200.build [--force] [--verbose]

The library links the CUDA runtime statically, so loading it needs neither a
GPU nor libcudart on the loader path; running it needs a B200."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmorello.so")
SOURCES = ["api.cu", "skinny.cu", "gemv_stream.cu", "gemm_tcgen05.cu", "f32_split.cu", "pad.cu", "selftest.cu", "tensormap.cu", "noalloc.cu",
           "linear_api.cu", "linear_tile.cu", "linear_rows.cu", "linear_aux.cu", "route.cu"]
HEADERS = [os.path.join(CSRC, "internal.h"), os.path.join(CSRC, "sm100.cuh"),
           os.path.join(CSRC, "tensormap.h"), os.path.join(CSRC, "linear.h"), os.path.join(CSRC, "route.h"),
           os.path.join(CSRC, "activation.cuh"), os.path.join(CSRC, "column_sums.cuh"),
           os.path.join(os.path.dirname(HERE), "include", "morello.h")]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
              "-cudart", "static"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + HEADERS + [os.path.abspath(__file__)]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((cmd, subprocess.Popen(cmd)))
        objs.append(obj)
    for cmd, proc in procs:
        if proc.wait() != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    tmp = LIB + ".tmp.%d" % os.getpid()
    link = [_nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static",
            "-o", tmp, *objs]
    subprocess.run(link, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
