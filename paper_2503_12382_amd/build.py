"""Builds libreno.so (the HIP kernels for gfx950 and the C ABI) in place.

Every HIP source is compiled for gfx950 only, with packed-fp32 instruction
selection disabled, then linked with the host rANS coder into one shared
library next to this file.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libreno.so")
ARCH = "gfx950"

HIP_SOURCES = ["k_prep.hip", "k_dec.hip", "k_model.hip", "k_post.hip", "k_code.hip", "k_head.hip",
               "k_head_narrow.hip", "k_top.hip", "k_sample.hip", "k_step.hip", "api.cpp", "frame.cpp", "head.cpp", "step.cpp"]
HOST_SOURCES = ["rans.cpp"]
HEADERS = ["dev.h", "ctx.h", "head.h", "head_dev.h", "gemm.h", "logits.h", "step.h"]


def hipcc() -> str:
    for cand in (os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc"),
                 shutil.which("hipcc") or ""):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: the HIP library cannot be built")


def _flags():
    return ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", f"-I{os.path.join(ROOT, 'include')}"]


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    if src in HOST_SOURCES:
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", "-c",
               os.path.join(CSRC, src), "-o", obj, f"-I{os.path.join(ROOT, 'include')}"]
    else:
        lang = ["-x", "hip"] if src.endswith(".cpp") else []
        cmd = [hipcc()] + _flags() + lang + ["-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile of {src} failed:\n{r.stdout}\n{r.stderr}")
    msg = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if msg.strip() and verbose:
        print(msg, file=sys.stderr)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = HIP_SOURCES + HOST_SOURCES
    with cf.ThreadPoolExecutor(max_workers=min(len(srcs), 8)) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    tmp = LIB + ".tmp"
    cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
