"""Builds libonela.so (HIP, gfx950 only) in-tree with hipcc.

    python -m paper_2609_12399_amd.build

Every HIP translation unit is compiled for gfx950 with packed-fp32
instructions disabled, then linked into one shared library next to this file.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
OUT = os.path.join(HERE, "libonela.so")
BUILD_DIR = os.path.join(ROOT, "_build")
SOURCES = ["host_plan.cpp", "onela_api.cpp", "kernels_records.hip", "kernel_decode.hip", "kernel_replay.hip",
           "kernels_fullstate.hip", "kernels_select.hip", "kernels_prefill.hip",
           "kernels_delta.hip", "kernels_delta_prep.hip", "kernels_delta_scan.hip",
           "kernels_delta_reverse.hip", "kernels_delta_grad.hip", "kernel_delta_step.hip", "kernel_norm_rope.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include")]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    # the API calls the HIP runtime; host_plan.cpp is plain C++ (no HIP)
    lang = ["-x", "hip"] if src == "onela_api.cpp" else []
    cmd = [HIPCC, *FLAGS, *lang, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    """Compile every source and link libonela.so; returns its path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = OUT + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, OUT)
    if verbose:
        print(f"built {OUT}")
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
