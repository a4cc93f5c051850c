"""Compile libtriattn.so (HIP, gfx950) in-tree.

Usage: ``python -m paper_2507_21526_amd.build``.  The library is written next
to this file; the binding loads it from there.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libtriattn.so")
SOURCES = [os.path.join(CSRC, "triattn_schedule.cpp"),
           os.path.join(CSRC, "triattn_fwd.hip"),
           os.path.join(CSRC, "triattn_probe.hip"),
           os.path.join(CSRC, "triattn_scored.hip"),
           os.path.join(CSRC, "triattn_cache.hip"),
           os.path.join(CSRC, "triattn_paged.hip")]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"


def command(out: str):
    return [HIPCC, f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
            "-shared", "-Wall",
            # never emit packed fp32 VALU ops
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            "-o", out] + SOURCES


def build(verbose: bool = False) -> str:
    tmp = LIB + ".tmp"
    cmd = command(tmp)
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
