"""Builds the gfx950 shared library (hipcc, in-tree)."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmoe_ffn.so")
SOURCES = [os.path.join(HERE, "csrc", "moe_ffn.hip")]                                        # the layer
BLOCK_SOURCES = [os.path.join(HERE, "csrc", n) for n in ("block_ops.hip", "experts_w4.hip")]   # the operators around it

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # hipcc -O3 may otherwise form packed-fp32 VALU ops from scalar float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def build_library(verbose: bool = False, out: str = LIB_PATH, defines=()) -> str:
    """Compile csrc/*.hip, side by side, into libmoe_ffn.so next to this file; returns its path."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)

    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(4) as pool:
        sources = [*SOURCES, *BLOCK_SOURCES]
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in sources]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        list(pool.map(run, [[hipcc, *compile_flags, *defines, "-c", s, "-o", o] for s, o in zip(sources, objects)]))
        run([hipcc, *HIPCC_FLAGS, *objects, "-o", out])
    return out


if __name__ == "__main__":
    print(build_library(verbose=True))
