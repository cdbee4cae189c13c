"""The prompt kernel's index functions at the largest accepted sizes, compiled for the host from its own header."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_largest_sizes(tmp_path):
    exe = tmp_path / "attention_limits"
    # sums past an int's range are wrong even where they happen to wrap: they end the program
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler",
                           "-fsanitize=signed-integer-overflow,-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "paper_2608_02611_b200", "csrc"),
                           os.path.join(ROOT, "tests", "c", "attention_limits.cu"), "-o", str(exe), "-lubsan"], capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0 and done.stdout == "ok\n", done.stdout + done.stderr
