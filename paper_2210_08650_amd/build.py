"""Compile libhapi.so (HIP kernels + host runtime) for gfx950 with hipcc.

Objects go to ``_build/`` next to this file; the shared library lands in the
package directory so that it is found (and shipped) in-tree.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libhapi.so")
ARCH = os.environ.get("HAPI_OFFLOAD_ARCH", "gfx950")

SOURCES = ["conv.hip", "conv3x3.hip", "conv_first.hip", "stem.hip", "attention.hip", "elementwise.hip", "bottleneck.hip", "conv_pp.hip", "conv_f32.hip",
           "norm.hip", "head.hip", "gradients.hip", "rotary.hip", "cross_attention.hip", "cross_attention_back.hip", "api.cpp", "split.cpp", "tail.cpp", "block.cpp"]
HEADERS = [os.path.join(CSRC, "internal.h"), os.path.join(CSRC, "gemm_util.h"), os.path.join(CSRC, "tail.h"), os.path.join(CSRC, "block.h"), os.path.join(CSRC, "attend.h"), os.path.join(CSRC, "host_checks.h"),
           os.path.join(ROOT, "include", "hapi.h")]


def _hipcc() -> str:
    for c in ("/opt/rocm/bin/hipcc", shutil.which("hipcc") or ""):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found: the HIP toolchain is required to build libhapi")


def _flags() -> list:
    return ["-x", "hip", f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-Wall", "-Wno-unused-function", "-Wno-unused-result"]


def _compile(src: str) -> str:
    out = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc()] + _flags() + ["-c", os.path.join(CSRC, src), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stderr}")
    return out


def build(verbose: bool = False) -> str:
    """Compile every source (always) and link libhapi.so."""
    os.makedirs(OBJ, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
