"""The index functions that the attention kernels call, compiled for the host from the kernels' own headers
(tests/c/attention_index.cu) and checked there: a change of them shows without a GPU."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_02611_b200", "csrc")


def run(tmp_path, csrc):
    exe = tmp_path / "attention_index"
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", str(csrc),
                           os.path.join(ROOT, "tests", "c", "attention_index.cu"), "-o", str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)


def test_index_functions_of_the_kernels(tmp_path):
    done = run(tmp_path, CSRC)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout


@pytest.mark.parametrize("header,have,want", [
    ("kb_paged.cuh", "return g ^ ((g & 1) << 2);", "return g ^ ((g & 1) << 1);"),
    ("kb_paged.cuh", "return u < bigger ? u / (size + 1) : more + (u - bigger) / size;", "return u / (size + 1);"),
    ("kb_prompt.cuh", "const int seen = (int)(row + 1) + (int)nk - (int)nq;", "const int seen = (int)row + (int)nk - (int)nq;"),
    ("kb_rope.cuh", "const double part = t - floor(t);", "const double part = t - (double)(long long)t;"),
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


def test_registers_of_the_kernels_of_prompts(tmp_path):
    """Their warpgroups split 96 registers per thread, which is what the compiler has to launch them with, and the
    loops of the exponentials must not spill."""
    from paper_2608_02611_b200 import build
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "-ldl", "--threads=2")]
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), *flags, "-Xptxas", "-v", "-I", CSRC, "-c",
                           os.path.join(ROOT, "tests", "c", "attention_kernels.cu"), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    text = done.stdout + done.stderr
    assert text.count("Used 96 registers") == 4, text
    spills = [int(n) for n in re.findall(r"(\d+) bytes spill stores", text)]
    assert max(spills) <= 64, spills     # a few words of the warp that hands out the items


def test_header_is_plain_c99(tmp_path):
    from paper_2608_02611_b200 import build
    lib_path = build.build()
    src = tmp_path / "use.c"
    src.write_text('#include "kb_attention.h"\n'
                   "int main(void) {\n"
                   "  kb_ctx* ctx = 0;\n"
                   "  kb_paged_cache cache = {0, 0, 8, 8, 8, 8, 8, 8, 1, 16};\n"
                   "  if (kb_ctx_create(0, &ctx) == KB_OK) {\n"
                   "    (void)kb_attention_paged(ctx, 0, 8, 8, 1, &cache, 1, 8, KB_F16, 0, 0, 0, 0, 0, 1.0f, 0, 8, 8, 0, 0);\n"
                   "    kb_ctx_destroy(ctx);\n"
                   "  }\n"
                   "  return 0;\n"
                   "}\n")
    done = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), lib_path, "-o",
                           str(tmp_path / "use"), "-Wl,-rpath," + os.path.dirname(lib_path), "-Wl,--allow-shlib-undefined"],
                          capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
