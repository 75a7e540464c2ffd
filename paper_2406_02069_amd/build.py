"""Compiles the HIP sources under csrc/ into libpkv.so (gfx950 only), in-tree."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libpkv.so")
SOURCES = ["pkv_api.hip", "pkv_score.hip", "pkv_resident.hip", "pkv_stream.hip", "pkv_lag.hip", "pkv_sift.hip", "pkv_sweep.hip", "pkv_select.hip", "pkv_gather.hip", "pkv_decode.hip",
           "pkv_rotary.hip", "pkv_decode_long.hip", "pkv_prefill.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wno-unused-result",
    # packed fp32 VALU forms are kept out of the generated code on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


def build(verbose: bool = False, extra_flags=(), out: str = LIB) -> str:
    cmd = [HIPCC] + FLAGS + list(extra_flags) + [os.path.join(CSRC, s) for s in SOURCES] + ["-o", out]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    return out


if __name__ == "__main__":
    build(verbose=True)
    print("built", LIB)
    sys.exit(0)
