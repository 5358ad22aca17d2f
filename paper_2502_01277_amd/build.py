"""Build libocto.so (HIP, gfx950) in-tree: python -m paper_2502_01277_amd.build"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libocto.so")
SOURCES = ["conv_bf16.hip", "conv_f16.hip", "conv_flow_bf16.hip", "conv_flow_f16.hip", "conv_flow_f8.hip", "conv_small_bf16.hip", "conv_small_f16.hip", "conv_small_f32.hip", "conv_f32.hip", "conv_f8.hip", "conv.hip", "stem.hip", "entry.hip", "block.hip", "lead.hip", "conv1x1.hip", "glue.hip", "preproc.hip", "postproc.hip", "pipeline.hip", "ops_api.hip", "probes.hip", "executor.hip", "attend_f16.hip", "attend_bf16.hip", "attend_f32.hip", "attend_tile_f16.hip", "attend_tile_bf16.hip", "attend.hip", "rotate.hip", "cache4.hip", "norm.hip", "product_bf16.hip", "product_f16.hip", "product_f32.hip", "product_f8.hip", "product.hip", "sample.hip", "sched.cpp", "runtime.cpp", "placement.cpp"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-result", "-Wno-unused-value"]


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, "_build", os.path.splitext(src)[0] + ".o")
    os.makedirs(os.path.dirname(obj), exist_ok=True)
    cmd = ["hipcc", *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(verbose: bool = True) -> str:
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", OUT, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print("built", OUT)
    return OUT


if __name__ == "__main__":
    build()
