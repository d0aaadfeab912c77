"""Builds the gfx950 shared library ``libexflow_moe.so`` in-tree with hipcc.

Usage: ``python -m paper_2401_08383_amd.build``.  Cross-compiles without a GPU.
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(CSRC, "_build")
LIB = os.path.join(PKG, "libexflow_moe.so")
SOURCES = ["api.hip", "gate.hip", "dispatch.hip", "ffn.hip", "ffn_keep.hip", "ffn_stream.hip", "combine.hip", "layer.hip", "affinity.hip", "affinity_direct.hip", "placement.hip", "probe.hip", "ffn_once.hip", "ffn_once_second.hip", "ffn_routed.hip", 
           "product.hip", "product_forward.hip", "product_rows_gradient.hip", "product_weight_gradient.hip", "product_mx4_tiles.hip", "product_mx4.hip",
           "product_exact.hip", "mx4.hip", "route.hip", "rows.hip", "q4.hip", "product_q4.hip", "product_q4_stream.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 VALU forms are kept off (device pass only; the host pass ignores the feature)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-function", "-Wno-pass-failed",
    "-mllvm", "-pragma-unroll-threshold=1000000",  # the K loops are unrolled by hand-placed slots: completely or not at all
]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in res.stderr.splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as pool:
        objs = list(pool.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
