"""Builds libspp.so (the HIP kernels and the C interface) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libspp.so")
SOURCES = ["spp_api.hip", "spp_pool.hip", "spp_radix.hip", "spp_graph.hip", "spp_vip.hip", "spp_sample.hip",
           "spp_gather.hip", "spp_cache.hip", "spp_local.hip", "spp_mx4.hip", "spp_layer.hip", "spp_grad.hip", "spp_adamw.hip",
           "spp_fp8.hip", "spp_hidden.hip", "spp_gated.hip", "spp_gated_grad.hip", "spp_fp8_grad.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc", "-Wall",
         # no packed-fp32 code generation on the device.  hipcc hands the option to both of its passes:
         # the gfx950 pass honours it, the x86 host pass prints "not a recognized feature for this
         # target (ignoring feature)", which is about the host only (tests/test_boundary_cpu.py shows
         # the effect on the device pass alone).
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-ffp-contract=off"]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    subprocess.check_call([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs])
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
