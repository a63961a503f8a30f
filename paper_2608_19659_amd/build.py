"""Build step for libfleetsieve: compiles the gfx950 kernels and the C-ABI
host runtime into ``paper_2608_19659_amd/libfleetsieve.so`` with hipcc.

Flags that matter for the numerics: no fused multiply-add contraction and no
fast-math, so every binary32 multiply and every quotient rounds exactly as
the C ABI documents.  Packed FP32 instructions are disabled."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libfleetsieve.so")
SOURCES = [os.path.join(CSRC, n) for n in ("fs_kernels.hip", "fs_linear.hip", "fs_cache.hip", "fs_attention.hip",
                                           "fs_api.cpp", "fs_serving_api.cpp")]

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    "-I", INCLUDE, "-I", CSRC,
]


def hipcc() -> str:
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def build_library(extra_flags=(), out: str = LIB, verbose: bool = False) -> str:
    """Compile libfleetsieve.so (always recompiles; the sources side by side)."""
    tmp = out + ".tmp"
    with tempfile.TemporaryDirectory(prefix="fleetsieve_") as work:
        objects = [os.path.join(work, os.path.basename(src) + ".o") for src in SOURCES]
        compiles = [[hipcc(), *HIP_FLAGS, *extra_flags, "-c", src, "-o", obj] for src, obj in zip(SOURCES, objects)]
        link = [hipcc(), *HIP_FLAGS, *extra_flags, "-shared", *objects, "-o", tmp]
        if verbose:
            for cmd in (*compiles, link):
                print(" ".join(cmd), file=sys.stderr)
        with ThreadPoolExecutor(max_workers=4) as pool:
            list(pool.map(lambda cmd: subprocess.run(cmd, check=True, cwd=HERE), compiles))
        subprocess.run(link, check=True, cwd=HERE)
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build_library(verbose=True))
