"""Compile the HIP sources in csrc/ into libcfdetr.so (gfx950), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcfdetr.so")
SOURCES = ["api.hip", "select.hip", "roi.hip", "rowwise.hip", "gemm.hip", "layer.hip", "small_layer.hip",
           "few_rows.hip", "attention.hip", "sched.hip", "rotary.hip", "diff_attention.hip", "diff_tiles.hip",
           "norm_residual.hip", "memory_advance.hip", "memory_rows.hip", "memory_attention.hip"]
# A kernel's first 14 words of arguments come in scalar registers with the launch, so that its first
# loads need not wait for a load of their addresses (arguments that are structs are left in memory).
FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-fvisibility=hidden",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-mllvm", "-amdgpu-kernarg-preload-count=16"]
# Per-source extras.  The attention kernels read every MFMA result back for the
# softmax, so its accumulators should live in ordinary VGPRs (no AGPR copies); the
# GEMMs only read theirs in the epilogue and are faster with AGPR accumulators.
EXTRA_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "diff_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "diff_tiles.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "memory_attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def build(verbose: bool = True) -> str:
    """Compile every source and link the shared library; returns its path."""
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    hipcc = _hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, *EXTRA_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{res.stdout}\n{res.stderr}")
        return obj

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), 8)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    if verbose:
        print(f"built {LIB}", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
