"""Compiles the HIP library for gfx950 with hipcc (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libflashdp.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def sources():
    return [os.path.join(CSRC, "flashdp_api.hip"), os.path.join(CSRC, "flashdp_layers.hip")]


def build_library(verbose: bool = False, extra_flags=()) -> str:
    """Compiles the sources side by side and links them."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)
        if verbose and res.stderr.strip():
            print(res.stderr)

    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor() as pool:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources()]
        list(pool.map(lambda so: run([hipcc, *HIPCC_FLAGS, *extra_flags, "-c", "-o", so[1], so[0]]), zip(sources(), objects)))
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB_PATH, *objects])
    return LIB_PATH


if __name__ == "__main__":
    print(build_library(verbose=True))
