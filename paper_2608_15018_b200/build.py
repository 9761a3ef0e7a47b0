"""Compile the CUDA library in-tree for sm_100a with nvcc (no GPU needed)."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libs2moe.so")
SOURCES = ["s2moe_api.cu", "attn_api.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--use_fast_math", "-Xcompiler", "-fPIC",
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps.append(os.path.join(os.path.dirname(HERE), "include", "s2moe.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Build ``libs2moe.so`` next to this file if it is missing or out of date."""
    if force or _stale():
        # one object per source, compiled beside each other
        with tempfile.TemporaryDirectory() as tmp:
            objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
            base = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else [])
            running = [subprocess.Popen(base + ["-c", os.path.join(CSRC, s), "-o", o]) for s, o in zip(SOURCES, objects)]
            for p in running:
                p.wait()
            for p in running:
                if p.returncode:
                    raise subprocess.CalledProcessError(p.returncode, p.args)
            subprocess.check_call([_nvcc()] + NVCC_FLAGS + ["-shared", "-o", LIB] + objects)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
