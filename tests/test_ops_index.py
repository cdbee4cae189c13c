"""The index functions that the model operators' kernels call, compiled for the host from the kernels' own
headers (tests/c/ops_index.cu) and checked there: a change of them shows without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_02611_b200", "csrc")


def run(tmp_path, csrc):
    exe = tmp_path / "ops_index"
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", str(csrc),
                           os.path.join(ROOT, "tests", "c", "ops_index.cu"), "-o", str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)


def test_index_functions_of_the_kernels(tmp_path):
    done = run(tmp_path, CSRC)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout


@pytest.mark.parametrize("header,have,want", [
    ("kb_matmul.cuh", "tn = r / h;", "tn = r / (h + 1);"),
    ("kb_matmul.cuh", "return (groups * o + splits - 1) / splits;", "return (groups * o) / splits;"),
    ("kb_quant.cuh", "((k ^ (r >> 3)) & 15) * 8", "((k ^ (r >> 4)) & 15) * 8"),
    ("kb_block8.cuh", "lane * 8 + j : j * 32 + lane", "lane * 8 + j : j * 16 + lane"),
])
def test_a_changed_index_is_noticed(tmp_path, header, have, want):
    """A mistake planted in a copy of a header makes the check fail."""
    copy = tmp_path / "pkg" / "csrc"
    copy.mkdir(parents=True)
    include = tmp_path / "include"
    include.mkdir()
    for src, dst in ((CSRC, copy), (os.path.join(ROOT, "include"), include)):
        for name in os.listdir(src):
            if name.endswith((".h", ".cuh")):
                text = open(os.path.join(src, name)).read()
                if name == header:
                    assert text.count(have) == 1
                    text = text.replace(have, want)
                (dst / name).write_text(text)
    assert run(tmp_path, copy).returncode == 1


def test_registers_of_the_kernel_of_cta_pairs(tmp_path):
    """Its warps split 168 registers per thread, which is what the compiler has to launch it with; and its
    sums leave none over: spills in its loop cost a fifth of its speed."""
    from paper_2608_02611_b200 import build
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "-ldl", "--threads=2")]
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), *flags, "-Xptxas", "-v", "-I", CSRC, "-c",
                           os.path.join(ROOT, "tests", "c", "pair_kernel.cu"), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    text = done.stdout + done.stderr
    assert text.count("Used 168 registers") == 2, text
    assert text.count("0 bytes spill stores, 0 bytes spill loads") == 2, text
