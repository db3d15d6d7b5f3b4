"""Compile the HIP library (libblockgtq.so) in-tree for gfx950 with hipcc."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libblockgtq.so")
BUILD_DIR = os.path.join(ROOT, "_build")
SOURCES = ["blockgtq.cpp", "kernels.hip", "decode_f16.hip", "prefill.hip", "window.hip", "step.hip", "probe.hip", "quantize.hip", "noalloc.hip", "rows.hip", "cross.hip", "cross_tile_bf16.hip", "cross_tile_fp32.hip", "norm_rope.hip", "paged.hip", "paged_quantize.hip", "paged_tile_bf16.hip", "paged_tile_fp32.hip"] + [f"{k}_bv{b}.hip" for k in ("decode", "cross", "paged", "paged_decode") for b in range(1, 9)]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed fp32 instructions anywhere in the device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
    "-Wall", "-Wno-unused-function",
]
# The decode kernels compare softmax scores with max(): no NaN can reach them
# (finite codebooks and radii, -inf only as a mask), so skip the IEEE
# canonicalization that would otherwise precede every max.
DECODE_FLAGS = ["-fno-honor-nans", "-mno-amdgpu-ieee"]
# rows.hip indexes a key row's words at a wave-uniform position and keeps rows of
# up to 16 words in registers (no scratch): beside its accumulators the default
# budget (bytes) puts the array in scratch memory.  The 32-word kernels keep it
# there all the same (176 bytes a lane), as do those of cross_impl.h without the
# flag (0 to 164 bytes of spilled registers up to 16 words, 304 to 416 above).
INDEXED_FLAGS = ["-mllvm", "-amdgpu-promote-alloca-to-vector-limit=100000"]


def _run(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("build failed: " + " ".join(cmd))
    return r


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    objs = []
    cmds = []
    for src in SOURCES:
        obj = os.path.join(BUILD_DIR, src + ".o")
        lang = ["-x", "hip"]
        extra = DECODE_FLAGS if src.startswith("decode_") else INDEXED_FLAGS if src == "rows.hip" else []
        cmds.append([HIPCC, *FLAGS, *extra, *lang, "-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    with ThreadPoolExecutor(max_workers=min(len(cmds), os.cpu_count() or 4, 16)) as ex:
        list(ex.map(_run, cmds))
    tmp = OUT + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp])
    os.replace(tmp, OUT)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
