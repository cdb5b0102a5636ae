"""Builds the gfx950 shared libraries (libpf.so, libpf_layer.so) in-tree with hipcc.

`python -m paper_2504_00492_amd.build` or `build_library()`.  Cross-compiles without a GPU.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpf.so")
# the operators around the delta rule, a library of their own: who runs the recurrence alone does not load them
LAYER_LIB = os.path.join(HERE, "libpf_layer.so")
LAYER_SOURCES = ["pf_layer_api.hip", "pf_norm.hip", "pf_quant.hip", "pf_matmul.hip", "pf_gated.hip", "pf_heads.hip",
                 "pf_gdelta_flow.hip", "pf_gdelta_scan.hip", "pf_gdelta_grad.hip", "pf_gdelta_step.hip"]
SOURCES = ["pf_api.hip", "pf_generic.hip", "pf_flow.hip", "pf_scan.hip", "pf_fused.hip", "pf_segments.hip", "pf_sigdelta.hip", "pf_rescale.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Packed-fp32 VALU forms are switched off for every kernel of this library.  The feature flag
# reaches the host pass as well (hipcc has no way to hand a flag with an argument to the device
# pass alone); the host pass does not know the feature and says so once per translation unit,
# which is harmless: _compile drops exactly that line from what it passes on.
HOST_PASS_NOTE = "'-packed-fp32-ops' is not a recognized feature for this target"
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-value",
         "-Wno-unknown-warning-option",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    obj = os.path.join(CSRC, src.replace(".hip", ".o"))
    run = subprocess.run([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj], stderr=subprocess.PIPE, text=True)
    noise = [ln for ln in run.stderr.splitlines() if ln.strip() and HOST_PASS_NOTE not in ln]
    if noise:
        print("\n".join(noise), file=sys.stderr)
    if run.returncode != 0:
        raise subprocess.CalledProcessError(run.returncode, run.args)
    return obj


def build_library(verbose: bool = False) -> str:
    """Compile every source and link libpf.so and libpf_layer.so.  Always recompiles."""
    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(_compile, SOURCES + LAYER_SOURCES))
    link = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC"]
    subprocess.run([*link, "-o", LIB, *objs[:len(SOURCES)]], check=True)
    subprocess.run([*link, "-o", LAYER_LIB, *objs[len(SOURCES):], "-L" + HERE, "-lpf", "-Wl,-rpath,$ORIGIN"], check=True)
    if verbose:
        print("built", LIB, "and", LAYER_LIB, file=sys.stderr)
    return LIB


def library_path() -> str:
    return LIB


if __name__ == "__main__":
    build_library(verbose=True)
