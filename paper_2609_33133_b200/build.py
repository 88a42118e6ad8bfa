"""Builds libaugtree.so (sm_100a, nvcc) and _marshal.*.so (g++, torch's headers) in-tree.  `python -m paper_2609_33133_b200.build`.

The second one takes the arguments of binding.Block apart and fits one Python and one torch alone, so their versions are in its name: under others it is
missing and is built again."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaugtree.so")


def marshal_path() -> str:
    import torch
    return os.path.join(HERE, f"_marshal.{sys.implementation.cache_tag}.torch-{torch.__version__}.so")


CUDA = "/usr/local/cuda"
SOURCES = ["augtree.cu", "lm.cu", "block.cu", "plan.cpp", "planner.cpp"]
HEADERS = ["ptx.cuh", "fwd_kernel.cuh", "bwd_kernel.cuh", "dq_kernel.cuh", "dql_kernel.cuh", "pair_tile.cuh", "lm_tile_kernel.cuh", "lm_few_kernel.cuh", "lm_kernels.cuh", "ckpt.cuh", "act_kernels.cuh",
           "block_kernels.cuh", "wgrad_kernel.cuh", "handle.h", "launch.h", "plan.h", os.path.join("..", "..", "include", "augtree.h")]
MARSHAL_SOURCES = ["marshal.cpp", os.path.join("..", "..", "include", "augtree.h")]


def _stale(target, sources) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in sources)


def _start_marshal():
    """g++ on the argument marshalling of binding.Block, against the headers of the torch that runs it."""
    import torch
    at = os.path.dirname(torch.__file__)
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I" + os.path.join(at, "include"),
           "-I" + os.path.join(at, "include", "torch", "csrc", "api", "include"), "-I" + sysconfig.get_paths()["include"], "-I" + CUDA + "/include",
           "-o", marshal_path(), os.path.join(CSRC, MARSHAL_SOURCES[0]), "-L" + os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def build(force: bool = False, verbose: bool = False) -> str:
    marshal = _start_marshal() if force or _stale(marshal_path(), MARSHAL_SOURCES) else None
    failed = []
    if force or _stale(LIB, SOURCES + HEADERS):
        nvcc = os.environ.get("NVCC", CUDA + "/bin/nvcc")
        cmd = [nvcc, "--threads", "0", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
               "-Xcompiler", "-fPIC", "-cudart", "static",
               "-o", LIB] + [os.path.join(CSRC, f) for f in SOURCES]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
            failed.append("nvcc failed building libaugtree.so")
        elif verbose:
            sys.stderr.write(res.stderr)
    if marshal is not None:
        out = marshal.communicate()[0]
        if marshal.returncode != 0:
            sys.stderr.write(out)
            failed.append("the C++ compiler failed building " + os.path.basename(marshal_path()))
    if failed:
        raise RuntimeError("; ".join(failed))
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
