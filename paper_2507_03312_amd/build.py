"""Build libmpx.so (the HIP library behind include/mpx.h) for gfx950.

Each .hip source under csrc/ is compiled with hipcc for gfx950 and the
objects are linked into paper_2507_03312_amd/libmpx.so.  Run as
``python -m paper_2507_03312_amd.build``.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libmpx.so")
BUILD_DIR = os.path.join(PKG, "_build")
SOURCES = ["gemm_f16.hip", "gemm_bf16.hip", "gemm_staged_f16.hip", "gemm_staged_bf16.hip",
           "gemm_wide_f16.hip", "gemm_wide_bf16.hip", "support.hip", "attention.hip", "sweep.hip",
           "gemm_act8_f16.hip", "gemm_act8_bf16.hip",
           "gated_f16.hip", "gated_bf16.hip", "linear_ce_f16.hip", "linear_ce_bf16.hip",
           "linear_ce_pair_f16.hip", "linear_ce_pair_bf16.hip",
           "gemm.hip", "gemm_f32.hip", "support_f32.hip", "act8.hip", "rope.hip", "logprob.hip",
           "gated.hip", "linear_ce.hip", "qknorm_rope.hip", "dropout.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed float32 instructions (v_pk_*_f32) are generated: the kernels
    # are written and checked without them
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
