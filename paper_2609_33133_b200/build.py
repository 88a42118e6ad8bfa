"""Builds libaugtree.so (sm_100a) in-tree with nvcc.  `python -m paper_2609_33133_b200.build`."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaugtree.so")
SOURCES = ["augtree.cu", "lm.cu", "block.cu", "plan.cpp", "planner.cpp"]
HEADERS = ["ptx.cuh", "fwd_kernel.cuh", "bwd_kernel.cuh", "dq_kernel.cuh", "dql_kernel.cuh", "pair_tile.cuh", "lm_tile_kernel.cuh", "lm_few_kernel.cuh", "lm_kernels.cuh", "ckpt.cuh", "act_kernels.cuh",
           "block_kernels.cuh", "wgrad_kernel.cuh", "handle.h", "launch.h", "plan.h", os.path.join("..", "..", "include", "augtree.h")]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in SOURCES + HEADERS)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "--threads", "0", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
           "-Xcompiler", "-fPIC", "-cudart", "static",
           "-o", LIB] + [os.path.join(CSRC, f) for f in SOURCES]
    if verbose:
        cmd.insert(1, "-Xptxas")
        cmd.insert(2, "-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libaugtree.so")
    if verbose:
        sys.stderr.write(res.stderr)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
