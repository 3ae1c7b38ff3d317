"""Builds the HIP library in-tree (gfx950 only)."""
from __future__ import annotations

import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcompressed_layer.so")
SOURCES = ["compress.cpp", "huffman.cpp", "planner.cpp", "device.hip", "mx/quantize.hip", "mx/route.hip", "mx/product.hip",
           "f8/quantize.hip", "f8/norm.hip", "f8/product.hip"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared", "--offload-arch=gfx950",
    "-munsafe-fp-atomics",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build_library(verbose: bool = False) -> str:
    """Host sources go through g++, the kernels through hipcc, four at a time; hipcc links."""
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]

    def compile_one(s):
        obj = os.path.join(bdir, s.replace("/", "_") + ".o")
        if s.endswith(".hip"):
            _run([hipcc(), *[f for f in HIPCC_FLAGS if f != "-shared"], *inc, "-c", os.path.join(CSRC, s), "-o", obj], verbose)
        else:
            _run(["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", *inc, "-c", os.path.join(CSRC, s), "-o", obj], verbose)
        return obj

    with ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    _run([hipcc(), "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", LIB], verbose)
    return LIB


def library_is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(d, f) for d, _, fs in os.walk(CSRC) for f in fs] + [os.path.join(ROOT, "include", "compressed_layer.h")]
    return any(os.path.getmtime(d) > t for d in deps)


if __name__ == "__main__":
    print(build_library(verbose=True))
