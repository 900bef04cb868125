"""Builds the C-ABI library ``libgcn_admm.so`` in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = [os.path.join(HERE, "csrc", "gcn_admm.cu"), os.path.join(HERE, "csrc", "grouped.cu")]
HEADERS = [os.path.join(HERE, "csrc", "kernels.cuh"), os.path.join(HERE, "csrc", "gemm_half.cuh"), os.path.join(HERE, "csrc", "gemm_tc.cuh"), os.path.join(HERE, "csrc", "graph_index.hpp"), os.path.join(HERE, "csrc", "shard_plan.hpp"), os.path.join(HERE, "csrc", "memory.hpp"),
           os.path.join(HERE, "csrc", "grouped.hpp"), os.path.join(HERE, "csrc", "grouped_plan.hpp"), os.path.join(HERE, "csrc", "grouped_mma.cuh"), os.path.join(HERE, "csrc", "grouped_words.hpp"), os.path.join(HERE, "csrc", "tensor_map.hpp"),
           os.path.join(os.path.dirname(HERE), "include", "gcn_admm.h")]
LIB = os.path.join(HERE, "libgcn_admm.so")


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles the library when it is missing or older than its sources; returns its path."""
    if not force and not is_stale():
        return LIB
    cmd = [nvcc_path(), "-std=c++17", "-O3", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC,-fopenmp", "-shared", "-t", "0"]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += SOURCES + ["-o", LIB]
    proc = subprocess.run(cmd, capture_output=True, text=True)
    if proc.returncode != 0:
        raise RuntimeError("nvcc failed:\n" + proc.stdout + proc.stderr)
    if verbose:
        print(proc.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
