"""Builds libqgx.so (the C-ABI library) from csrc/ with hipcc for gfx950, in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqgx.so")
SOURCES = ["qgx_lib.hip", "qgx_tables.hip", "qgx_encode.hip", "qgx_decode.hip", "qgx_fit.hip", "qgx_game.hip", "qgx_metrics.hip",
           "qgx_clip.hip", "qgx_layer_norm.hip", "qgx_position_bias.hip"]

# -ffp-contract=off: the rounding decisions are specified as separately rounded binary32 operations.
# packed-fp32 ops are switched off for the device pass (the host pass warns that it ignores the flag).
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument"]


def build(verbose: bool = False, extra=()) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc, *FLAGS, *extra, "-shared", "-o", LIB + ".tmp"] + [os.path.join(CSRC, s) for s in SOURCES]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True, extra=sys.argv[1:])
    print("built", LIB)
