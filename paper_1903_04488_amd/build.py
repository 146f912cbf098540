"""Builds libcsketch.so (the C-ABI library of HIP kernels) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libcsketch.so")
SOURCES = ["cs_host.cpp", "cs_kernels.hip", "cs_lattice.hip", "cs_walk.hip", "cs_topk.hip", "cs_index.hip",
           "cs_norm.hip", "cs_token.hip", "cs_token_f32.hip", "cs_token_bf16.hip", "cs_token_f16.hip", "cs_adamw.hip"]

HIPCC_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-shared",
    "--offload-arch=gfx950",
    "-munsafe-fp-atomics",                      # fp32 atomic add as one hardware instruction
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument",
]


def build_library(verbose: bool = False) -> str:
    """One object a source, a few at a time (each compiler needs a core and half a gigabyte), then the library."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    jobs = max(1, min(8, os.cpu_count() or 1))

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        subprocess.check_call(cmd)

    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(jobs) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compile_flags = [f for f in HIPCC_FLAGS if f != "-shared"]
        # (the longest first)
        order = sorted(range(len(SOURCES)), key=lambda i: "walk" not in SOURCES[i] and "token_" not in SOURCES[i])
        list(pool.map(lambda i: run([hipcc, *compile_flags, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-x", "hip", "-c",
                                     os.path.join(CSRC, SOURCES[i]), "-o", objects[i]]), order))
        run([hipcc, *HIPCC_FLAGS, "-o", LIB, *objects])
    return LIB


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "csketch.h")]
    return any(os.path.getmtime(f) > t for f in deps)


if __name__ == "__main__":
    print(build_library(verbose=True))
