"""Build libemu.so (HIP for gfx950) in-tree.

    python -m paper_2609_04663_amd.build

Each .hip source is compiled with hipcc for gfx950 (packed-FP32 instruction
forms disabled) into ``_build/`` and linked into ``libemu.so`` next to this
file.  The build always recompiles.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libemu.so")
SOURCES = ["split.hip", "gemm_f32.hip", "gemm_f64.hip", "gemm_f64s.hip", "gemm_f64t.hip",
           "gemm_f64w.hip", "fallback.hip", "kbin.hip", "emu_api.hip", "moe_route.hip",
           "moe_combine.hip", "grouped.hip", "grouped16_gemm_bf16.hip",
           "grouped16_gemm_f16.hip", "grouped16_wgrad_bf16.hip", "grouped16_wgrad_f16.hip",
           "grouped_few.hip", "grouped_staged_f32.hip", "grouped_staged_bf16.hip",
           "grouped_staged_f16.hip", "q4.hip", "q4_f32.hip", "q4_bf16.hip", "q4_f16.hip",
           "moe_api.hip"]
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-I", os.path.join(HERE, "..", "include"), "-c",
           os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build() -> str:
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=" + ARCH, "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
    sys.exit(0)
