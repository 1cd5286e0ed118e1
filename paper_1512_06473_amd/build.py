"""Build libqcnn.so (the HIP kernels and the C ABI) in-tree for gfx950.

    python -m paper_1512_06473_amd.build        # or __graft_entry__.build()

Each source is compiled by hipcc in parallel, then linked into one shared
library next to this file.  Packed-fp32 VALU instructions are disabled for
every translation unit (-packed-fp32-ops), so the compiler never forms
v_pk_add_f32 / v_pk_mul_f32 / v_pk_fma_f32.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libqcnn.so")
ARCH = os.environ.get("QCNN_OFFLOAD_ARCH", "gfx950")

SOURCES = ["dense_bf16.hip", "dense_f16.hip", "dense_f32.hip", "dense_api.cpp", "qcnn_api.cpp", "lut_build.hip", "conv_gather.hip", "conv_flat.hip", "conv_dense.hip", "conv_half.hip", "fc_few.hip", "fc_gather.hip", "fc_tiled.hip", "glue.hip", "quantize.hip", "ec_fc.hip", "ec_conv.hip", "scratch.cpp", "noalloc.hip", "peaks.hip"]

CXXFLAGS = [
    "-x", "hip", "--offload-arch=" + ARCH, "-O3", "-fPIC", "-std=c++17",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-I", INCLUDE, "-I", CSRC,
]


def hipcc() -> str:
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    return os.path.join(rocm, "bin", "hipcc")


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc()] + CXXFLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    # hipcc's host pass does not know the packed-fp32 feature and says so; drop that line.
    noise = [l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l and l.strip()]
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, "\n".join(noise)))
    if noise:
        sys.stderr.write("\n".join(noise) + "\n")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    jobs = min(len(SOURCES), max(1, min(16, os.cpu_count() or 1)))
    with cf.ThreadPoolExecutor(jobs) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc(), "--offload-arch=" + ARCH, "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout + r.stderr)
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
