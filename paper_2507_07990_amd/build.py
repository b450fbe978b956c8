"""Builds libsttm.so (HIP, gfx950) in-tree next to this file."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsttm.so")
SOURCES = ["sttm_api.hip", "sttm_spatial.hip", "sttm_temporal.hip", "sttm_reduce.hip", "sttm_rope.hip", "sttm_attention.hip",
           "sttm_evict.hip", "sttm_queries.hip", "sttm_queries_f32.hip", "sttm_queries_bf16.hip", "sttm_queries_f16.hip",
           "sttm_residual.hip"]
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",   # no packed-fp32 VALU forms
    "-fgpu-rdc" if False else "-fno-gpu-rdc",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = True) -> str:
    """(The sources one by one, side by side, then linked: none of them uses another's device code.)"""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as folder, ThreadPoolExecutor(min(len(SOURCES), 8, os.cpu_count() or 1)) as pool:
        def compiled(source: str) -> str:
            out = os.path.join(folder, source + ".o")
            cmd = [hipcc] + flags + ["-c", os.path.join(CSRC, source), "-o", out]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.run(cmd, check=True)
            return out
        objects = list(pool.map(compiled, SOURCES))
        cmd = [hipcc, "-shared", "--offload-arch=gfx950"] + objects + ["-o", LIB + ".part"]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    os.replace(LIB + ".part", LIB)                         # (in place only when it is whole)
    return LIB


if __name__ == "__main__":
    build()
    print("built", LIB)
