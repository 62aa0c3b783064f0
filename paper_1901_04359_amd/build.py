"""Builds the C-ABI library `libgtopk.so` for gfx950 with hipcc, in-tree.

    python -m paper_1901_04359_amd.build
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRCS = [os.path.join(PKG, "csrc", name)        # they include the *.hip.h kernel files beside them
        for name in ("gtopk.hip", "layer.hip")]
OUT = os.path.join(PKG, "libgtopk.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-fno-gpu-flush-denormals-to-zero", "-ffp-contract=off",
    # packed fp32 instructions are kept out of the generated code on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SRCS]
        cmds = [[hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-c", src, "-o", obj]
                for src, obj in zip(SRCS, objects)]
        if verbose:
            for cmd in cmds:
                print(" ".join(cmd), flush=True)
        running = [subprocess.Popen(cmd) for cmd in cmds]          # side by side
        codes = [p.wait() for p in running]
        for cmd, code in zip(cmds, codes):
            if code != 0:
                raise subprocess.CalledProcessError(code, cmd)
        link = [hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", OUT]
        if verbose:
            print(" ".join(link), flush=True)
        subprocess.run(link, check=True)
    return OUT


if __name__ == "__main__":
    build()
    sys.exit(0)
