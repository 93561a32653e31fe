"""Build libsoniq.so (gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libsoniq.so")
SOURCES = [os.path.join(HERE, "csrc", name) for name in (
    "soniq_kernels.hip", "soniq_api.cpp", "soniq_i8.hip", "soniq_kv.hip", "soniq_serve_api.cpp")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # IEEE fp32 in the quantizer and the epilogue: no contraction into FMA
    "-ffp-contract=off",
    # never emit packed fp32 arithmetic
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build(verbose: bool = False) -> str:
    """Compile every HIP source (side by side) into paper_2311_14114_amd/libsoniq.so."""
    with tempfile.TemporaryDirectory() as d:
        def compile_one(src):
            obj = os.path.join(d, os.path.basename(src) + ".o")
            _run(["hipcc", *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"),
                  "-I", os.path.join(HERE, "csrc"), "-c", src, "-o", obj], verbose)
            return obj

        with ThreadPoolExecutor(max_workers=4) as pool:
            objs = list(pool.map(compile_one, SOURCES))
        tmp = LIB + ".tmp"
        _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp], verbose)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
