"""Build librelaysum.so (HIP kernels + C ABI) for gfx950, in-tree.

    python -m paper_2110_04175_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "relaysum.hip")
SOURCES = [SRC, os.path.join(PKG, "csrc", "layer.hip")]
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "librelaysum.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# IEEE binary32 semantics on the device: no contraction into FMA, correctly
# rounded division, denormals kept; packed-FP32 instructions disabled.
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math",
    "-fhip-fp32-correctly-rounded-divide-sqrt", "-fno-gpu-flush-denormals-to-zero",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def build(verbose: bool = False, extra=()) -> str:
    """Compile the library (always recompiles) and return its path.  `extra`
    goes to every compilation and to the link."""
    tmp = LIB + ".tmp"
    # One process for each source, side by side; then the link.
    objects = [os.path.splitext(src)[0] + ".o" for src in SOURCES]
    running = []
    for src, obj in zip(SOURCES, objects):
        cmd = [HIPCC, *FLAGS, *extra, "-I", INCLUDE, "-c", "-o", obj, src]
        if verbose:
            print(" ".join(cmd), flush=True)
        running.append((cmd, subprocess.Popen(cmd, cwd=PKG)))
    for cmd, p in running:
        if p.wait() != 0:
            for _, other in running:
                other.wait()
            raise subprocess.CalledProcessError(p.returncode, cmd)
    cmd = [HIPCC, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", tmp, *objects, *extra]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True, cwd=PKG)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True, extra=sys.argv[1:])
