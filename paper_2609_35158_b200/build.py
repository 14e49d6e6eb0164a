"""Builds ``libpd.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libpd.so")
SOURCES = ["pd_api.cu", "pd_decode_attn.cu", "pd_decode_attn_fp8.cu", "pd_decode_attn_q4.cu", "pd_decode_attn_latent.cu", "pd_kv_append.cu", "pd_kv_expand_latent.cu", "pd_kv_q4.cu", "pd_rope.cu", "pd_rope_latent.cu", "pd_kv_transfer.cu", "pd_prefill_attn.cu", "pd_prefill_attn_d128.cu", "pd_prefill_attn_latent.cu", "pd_static.cu", "pd_decision.cu", "pd_pool.cu", "pd_probe.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
    "-Xcompiler", "-fPIC", "-shared", "--use_fast_math", "-Xptxas", "-v",
]


def _inputs():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))]
    inc = os.path.join(os.path.dirname(_HERE), "include")
    files += [os.path.join(inc, f) for f in os.listdir(inc) if f.endswith(".h")]
    return files


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(f) > t for f in _inputs())


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every CUDA source into ``libpd.so``; returns its path."""
    if not force and not is_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = f"{LIB}.{os.getpid()}.tmp"
    extra = os.environ.get("PD_NVCC_EXTRA", "").split()  # e.g. -DPD_ENABLE_TUNING for a profiling build
    cmd = [nvcc, *NVCC_FLAGS, *extra, *[os.path.join(CSRC, s) for s in SOURCES], "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed building libpd.so")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
