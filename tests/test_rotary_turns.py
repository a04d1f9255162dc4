"""Frequencies of rotary positions as fractions of a turn: the nearest multiple of 2^-64, compiled from the source by itself."""
import os
import re
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from paper_2412_12487_gb300 import build as B
from paper_2412_12487_gb300 import rotary_frequencies


def test_turns_are_rounded(tmp_path):
    """Within 1/2 of a unit, and what the second double of 1 / (2 pi) and the sums' roundings take: f 2^-55 by 2^-52, and
    2^-53 of the rest, which is below 2^11 units for frequencies of at most 1."""
    sympy = pytest.importorskip("sympy")
    text = open(os.path.join(B.CSRC, "echo_ops_rotary.cu")).read()
    body = re.search(r"uint64_t rotary_turns\(double f\) \{.*?\n\}\n", text, re.S).group(0)
    f = np.concatenate([rotary_frequencies(128), rotary_frequencies(80, base=500000.0, factor=8.0), rotary_frequencies(64, factor=32.0, length=4096),
                        [1.0, 0.1, 1e-4, -0.3, 1 / 3, 1e-9, -1e-9, 1e-15, 1e-19, 3e-20, 1e-25, 0.0]])
    src = tmp_path / "turns.cpp"
    src.write_text("#include <cmath>\n#include <cstdint>\n#include <cstdio>\n" + body + "int main() { const double f[] = {" +
                   ", ".join(float(x).hex() for x in f) + "}; for (double x : f) printf(\"%llu\\n\", (unsigned long long)rotary_turns(x)); }\n")
    exe = str(tmp_path / "turns")
    subprocess.run(["g++", "-std=c++17", "-ffp-contract=off", str(src), "-o", exe], check=True)
    got = [int(s) for s in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    turn = Fraction(str(sympy.N(1 / (2 * sympy.pi), 90)))
    for x, g in zip(f, got):
        off = (Fraction(g) - Fraction(float(x)) * turn * 2 ** 64) % 2 ** 64
        off = min(off, 2 ** 64 - off)
        assert off <= 0.5 + 2.0 ** -42 + abs(x) * 2.0 ** (64 - 55 - 52), (x, float(off))
