"""Build libwfstdec.so (HIP for gfx950) next to the Python binding.

Usage: python -m paper_1808_00687_amd.csrc.build   (or build() from Python)

Every source is compiled by hipcc for gfx950 only, with IEEE float32
arithmetic: no FP contraction, no fast-math, subnormals kept, and the packed
FP32 instructions disabled.
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(HERE)
ROOT = os.path.dirname(PKG)
INCLUDE = os.path.join(ROOT, "include")
OUT = os.path.join(PKG, "libwfstdec.so")
BUILD_DIR = os.path.join(PKG, "_build")

SOURCES = ["graph.cpp", "decode.cpp", "search_kernel.hip", "search_record_kernel.hip", "record_kernel.hip",
           "final_kernels.hip", "word_kernel.hip", "am.cpp", "am_norm.hip", "am_layer_norm.hip", "am_distill.hip", "am_clip.hip", "am_loglikes.hip", "am_linear.hip",
           "am_linear_bf16.hip", "am_linear_f16.hip", "am_linear_f8.hip", "am_gated.hip", "am_gated_bf16.hip",
           "am_gated_f16.hip", "am_gated_f8.hip"]
HEADERS = ["internal.h", "device_util.h", "record_set.h", "search_body.h", "am.h", "am_device.h", "am_linear.h", "am_places.h", "am_plan.h", "am_rows.h", "am_softmax.h", "am_thin.h", "am_tile.h"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++20",
    "-fPIC",
    "-ffp-contract=off",
    "-fno-fast-math",
    "-fno-gpu-flush-denormals-to-zero",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # atomics by one lane of a wave stay one instruction
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    "-Wall",
    "-I", INCLUDE,
    "-I", HERE,
]


def build(verbose: bool = False) -> str:
    """Compile every source (always) and link the shared library."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
        objs.append(obj)
        cmd = [HIPCC, "-x", "hip", *FLAGS, "-c", os.path.join(HERE, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        text = out.decode(errors="replace")
        # hipcc's host pass does not know the packed-fp32 feature: harmless
        lines = [l for l in text.splitlines() if "packed-fp32-ops" not in l and l.strip()]
        if lines and (verbose or p.returncode):
            print("\n".join(lines), file=sys.stderr)
        if p.returncode:
            failed.append(src)
    if failed:
        raise RuntimeError("hipcc failed on: " + ", ".join(failed))
    tmp = OUT + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs]
    subprocess.check_call(cmd)
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
