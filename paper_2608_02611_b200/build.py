"""Build the CUDA library in-tree:  python -m paper_2608_02611_b200.build

Two translation units (csrc/kb_host.cu: the gate, adjudication and selection; csrc/kb_ops.cu:
the model operators) compiled by nvcc for sm_100a into paper_2608_02611_b200/libkb.so, a plain
C-ABI shared library (include/kb.h, include/kb_ops.h); and csrc/kb_torch.cpp, compiled by g++ against
torch's headers into paper_2608_02611_b200/_kb_torch.so, the native half of the operators' binding.
The gate, and the operators from C, need only the former.
"""
from __future__ import annotations

import os
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libkb.so")
NATIVE = os.path.join(HERE, "_kb_torch.so")
NATIVE_SOURCE = os.path.join(CSRC, "kb_torch.cpp")
SOURCES = ["kb_host.cu", "kb_ops.cu"]
INCLUDE = os.path.join(HERE, "..", "include")

NVCC_FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-Wno-format-truncation", "-shared", "-ldl", "--threads=2",
]


def _newer(target: str, deps) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(f) > os.path.getmtime(target) for f in deps)


def _sources(*suffixes):
    return [os.path.join(d, f) for d in (CSRC, INCLUDE) for f in os.listdir(d) if f.endswith(suffixes)]


def stale() -> bool:
    return _newer(LIB, _sources(".cu", ".cuh", ".h"))


def native_marker() -> str:
    """What _kb_torch.so was compiled against, as it stands in the file and as its attribute ``built_for``."""
    import torch
    return f"torch {torch.__version__}, {sys.implementation.cache_tag}"


def native_stale() -> bool:
    """_kb_torch.so is missing, older than its sources, or compiled against another torch or Python."""
    if _newer(NATIVE, _sources(".h") + [NATIVE_SOURCE]):
        return True
    with open(NATIVE, "rb") as f:
        return native_marker().encode() + b"\0" not in f.read()


def build_native(force: bool = False) -> str:
    if force or native_stale():
        import sysconfig
        import torch
        from torch.utils import cpp_extension
        inc = cpp_extension.include_paths() + [os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"),
                                               sysconfig.get_paths()["include"]]
        libs = cpp_extension.library_paths()
        cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
        cmd += [f'-DKB_BUILT_FOR="{native_marker()}"']
        cmd += [f"-I{d}" for d in inc] + ["-o", NATIVE, NATIVE_SOURCE] + [f"-L{d}" for d in libs]
        cmd += ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda"]
        subprocess.run(cmd, check=True)
    return NATIVE


def build(force: bool = False, verbose: bool = False) -> str:
    if force or stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
              ["-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.run(cmd, check=True)
    try:
        build_native(force)
    except (OSError, subprocess.CalledProcessError, ImportError) as e:
        warnings.warn(f"{NATIVE} could not be built ({e}): the gate works without it, the operators' Python calls do not")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
