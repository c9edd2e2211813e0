"""Build libdc.so (HIP kernels for gfx950 + the C-ABI) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdc.so")
SOURCES = ["api.hip", "balance.hip", "balance_large.hip", "sort_large.hip", "advantage.hip", "plan.hip", "plan_large.hip", "plan_shards.hip", "gather.hip", "scatter.hip", "gae.hip", "noalloc.hip",
           "actor_api.hip", "logprob.hip", "embedding.hip", "embedding_grad.hip", "adamw.hip",
           "head_api.hip", "head_rows.hip", "head.hip", "head_grad.hip", "residual_norm.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-result"]


def build_lib(verbose: bool = False, extra: list[str] | None = None) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *FLAGS, *(extra or []), "-o", LIB, *[os.path.join(CSRC, s) for s in SOURCES]]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    build_lib(verbose=True, extra=sys.argv[1:])
