"""Builds the C-ABI library ``libmoe_hotpath.so`` from ``csrc/*.hip`` for gfx950.

Usage: ``python -m paper_2604_00785_amd.build`` (hipcc cross-compiles; no GPU needed).
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
LIB = os.path.join(PKG, "libmoe_hotpath.so")

# Packed-fp32 VALU forms are switched off on purpose for every HIP source.
HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++20", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def sources():
    return sorted(glob.glob(os.path.join(PKG, "csrc", "*.hip")))


def build(verbose: bool = True, extra=()) -> str:
    """Compiles the sources side by side (the products take minutes), then links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    include = ["-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc")]

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)

    with tempfile.TemporaryDirectory() as tmp:
        objects = {src: os.path.join(tmp, os.path.basename(src) + ".o") for src in sources()}
        with concurrent.futures.ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
            list(pool.map(lambda src: run([hipcc, *HIP_FLAGS, *extra, *include, "-c", "-o", objects[src], src]), objects))
        run([hipcc, *HIP_FLAGS, *extra, "-shared", "-o", LIB, *objects.values()])
    return LIB


if __name__ == "__main__":
    build(extra=sys.argv[1:])
