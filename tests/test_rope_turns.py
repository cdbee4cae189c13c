"""The part of a turn that the rotation takes per position (csrc/kb_rope.cuh, compiled for the host), against exact fractions:
what is off there is multiplied by the position."""
import os
import random
import subprocess
from fractions import Fraction

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798214808651")


def test_turns_per_position(tmp_path):
    exe = tmp_path / "rope_turns"
    done = subprocess.run([os.environ.get("NVCC", "nvcc"), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I",
                           os.path.join(ROOT, "paper_2608_02611_b200", "csrc"), os.path.join(ROOT, "tests", "c", "rope_turns.cu"), "-o", str(exe)],
                          capture_output=True, text=True)
    assert done.returncode == 0, done.stderr
    rng = random.Random(3)
    freqs = [0.0, 1.0, 0.25, 7.5, 2.25, 100.125, 3.141592653589793, 6.283185307179586, 2.0 ** -30, 1e-20, 5e-324, 1e-40, 12345.678, 65536.0]
    freqs += [1e4 ** (-i / 64) for i in range(64)] + [5e5 ** (-i / 32) for i in range(32)]
    freqs += [rng.uniform(1, 2) * 2.0 ** rng.randint(-70, 16) for _ in range(2000)]
    out = subprocess.run([str(exe)], input="\n".join(f.hex() for f in freqs), capture_output=True, text=True, timeout=60)
    lines = [line.split() for line in out.stdout.splitlines()]
    assert out.returncode == 0 and len(lines) == len(freqs)
    for f, (upper, rest) in zip(freqs, lines):
        want = Fraction(f) / TWO_PI
        off = (Fraction(int(upper), 1 << 64) + Fraction(float.fromhex(rest)) - want) % 1
        # the fraction is cut off behind 2^-64.  The rest is two numbers of at most 2^-54 of the quotient, or 2^-57 of the frequency,
        # taken with five roundings of 2^-24
        assert min(off, 1 - off) <= Fraction(1, 1 << 64) + Fraction(f) * Fraction(1, 1 << 76), f
