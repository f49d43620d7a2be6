"""Builds libboxconv.so (the HIP library behind include/boxconv.h) in-tree.

    python -m paper_1906_11367_amd.build

Every source is compiled for gfx950 with hipcc; packed-fp32 instructions are
disabled (-packed-fp32-ops).  Objects go to paper_1906_11367_amd/_build/.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libboxconv.so")
BUILD = os.path.join(PKG, "_build")
ARCH = "gfx950"

SOURCES = ["bc_api.cpp", "bc_block_norm.hip", "bc_box.hip", "bc_box_lds.hip", "bc_box_split.hip", "bc_linattn.hip", "bc_linattn_bf16.hip",
           "bc_linattn_f32.hip", "bc_mix.hip", "bc_mix_direct.hip",
           "bc_mix_i8.hip", "bc_mix_i8_few.hip", "bc_mix_i8_maps.hip", "bc_mix_pipe.hip", "bc_noalloc.hip", "bc_quant_i8.hip",
           "bc_scan.hip", "bc_scan_maps.hip", "bc_stream.hip"]


def hipcc() -> str:
    h = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(h):
        raise RuntimeError("hipcc not found (ROCm toolchain required to build libboxconv.so)")
    return h


def common_flags() -> list[str]:
    return ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [hipcc(), *common_flags(), "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    jobs = min(len(SOURCES), os.cpu_count() or 1)
    with cf.ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print(f"built {OUT}")
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
