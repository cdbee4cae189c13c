"""Build the CUDA library in-tree:  python -m paper_2608_02611_b200.build

Two translation units (csrc/kb_host.cu: the gate, adjudication and selection; csrc/kb_ops.cu:
the model operators) compiled by nvcc for sm_100a into paper_2608_02611_b200/libkb.so, a plain
C-ABI shared library (include/kb.h, include/kb_ops.h).
"""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkb.so")
SOURCES = ["kb_host.cu", "kb_ops.cu"]
INCLUDE = os.path.join(HERE, "..", "include")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-Wno-format-truncation", "-shared", "-ldl", "--threads=2",
]


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(d, f) for d in (CSRC, INCLUDE) for f in os.listdir(d) if f.endswith((".cu", ".cuh", ".h"))]
    return any(os.path.getmtime(f) > t for f in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if force or stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
              ["-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
