"""Compile libtriattn.so (HIP, gfx950) in-tree.

Usage: ``python -m paper_2507_21526_amd.build``.  The library is written next
to this file; the binding loads it from there.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

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


def command(source: str, out: str):
    return [HIPCC, f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall",
            # never emit packed fp32 VALU ops
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", os.path.join(ROOT, "include"), "-I", CSRC,
            "-c", source, "-o", out]


def build(verbose: bool = False) -> str:
    """The sources side by side (the longest takes minutes), then one library."""
    tmp = LIB + ".tmp"
    with tempfile.TemporaryDirectory(dir=PKG) as work:
        objects = [os.path.join(work, os.path.basename(s) + ".o") for s in SOURCES]

        def compile_one(source, out):
            cmd = command(source, out)
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.run(cmd, check=True)

        with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as pool:
            for done in [pool.submit(compile_one, s, o) for s, o in zip(SOURCES, objects)]:
                done.result()
        link = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp] + objects
        if verbose:
            print(" ".join(link), flush=True)
        subprocess.run(link, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
