"""CPU tests of the head's losses and rotary positions: what they do without a device or a context."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2412_12487_gb300 import build as B
from paper_2412_12487_gb300 import echo as E

OPS = {"echo_cross_entropy": E.CrossEntropyDesc, "echo_cross_entropy_grad": E.CrossEntropyGradDesc, "echo_distill": E.DistillDesc,
       "echo_distill_grad": E.DistillGradDesc, "echo_rotary": E.RotaryDesc, "echo_rotary_grad": E.RotaryDesc}


@pytest.mark.parametrize("name", sorted(OPS))
def test_no_context_is_refused(name):
    B.build()
    lib = E.load_library()
    assert getattr(lib, name)(None, C.byref(OPS[name]())) == 1
    assert getattr(lib, name)(None, None) == 1


def test_descriptors_are_the_header_s(tmp_path):
    """Sizes and offsets of the binding's structures against a C compiler's."""
    kinds = {"echo_cross_entropy_desc": E.CrossEntropyDesc, "echo_cross_entropy_grad_desc": E.CrossEntropyGradDesc, "echo_distill_desc": E.DistillDesc,
             "echo_distill_grad_desc": E.DistillGradDesc, "echo_rotary_desc": E.RotaryDesc}
    lines = []
    for c, py in kinds.items():
        lines.append(f'printf("{c} size %zu\\n", sizeof({c}));')
        lines += [f'printf("{c} {f} %zu\\n", offsetof({c}, {f}));' for f, _ in py._fields_]
    src = tmp_path / "offsets.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"echo.h\"\nint main(void) {\n" + "\n".join(lines) + "\nreturn 0;\n}\n")
    exe = str(tmp_path / "offsets")
    subprocess.run(["gcc", "-I", B.INCLUDE, str(src), "-o", exe], check=True)
    for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines():
        c, field, at = line.split()
        py = kinds[c]
        assert int(at) == (C.sizeof(py) if field == "size" else getattr(py, field).offset), line


def test_the_packed_descriptor_is_the_structure():
    d = E.RotaryDesc(1, 2, (3, 4), (5, 6), (7, 8), (9, 10), (11, 12), (13, 14), (15, 16), (17, 18), (19, 20), 21, 22, 23, 24, 25, 26, 27, 28, 29.5)
    assert E._ROTARY.pack(*range(1, 29), 29.5) == bytes(d)
    for form, kind, n, floats in ((E._CROSS_ENTROPY, E.CrossEntropyDesc, 15, 1), (E._DISTILL, E.DistillDesc, 20, 2)):
        values = list(range(1, n + 1 - floats)) + [0.5] * floats
        assert form.pack(*values) == bytes(kind(*values))
    with pytest.raises(E.EchoError):
        E._packed(E._CROSS_ENTROPY, 2 ** 70, *range(13), 1.0)


def test_heads_of_a_view():
    torch = pytest.importorskip("torch")
    x = torch.arange(2 * 3 * 4 * 6.0).view(2, 3, 4, 6)
    assert E._heads(x)[1:] == (2, 3, (72, 24, 6))
    assert E._heads(x[0])[1:] == (1, 3, (0, 24, 6)) and E._heads(x[0, 0])[1:] == (1, 1, (0, 0, 6))
    t = x.transpose(1, 2)
    assert E._heads(t)[0] is t and E._heads(t)[1:] == (2, 4, (72, 6, 24))
    assert E._heads(x[..., ::2])[0].is_contiguous()
    with pytest.raises(E.EchoError):
        E._heads(x[..., ::2], out=True)
    five = x.view(1, 2, 3, 4, 6)
    assert E._heads(five)[1:] == (1, 6, (0, 24, 6)) and E._heads(five, out=True)[0].data_ptr() == x.data_ptr()


def test_frequencies():
    f = E.rotary_frequencies(8, base=16.0)
    assert np.allclose(f, [1, 0.5, 0.25, 0.125], rtol=1e-15)
    assert np.allclose(E.rotary_frequencies(8, base=16.0, factor=4.0), f / 4, rtol=1e-15)
    length = 2 * np.pi * 8  # the pairs turn 8, 4, 2 and 1 times
    got = E.rotary_frequencies(8, base=16.0, factor=4.0, length=length, low=1, high=4)
    keep = np.array([1, 1, 1 / 3, 0])
    assert np.allclose(got, f * (keep + (1 - keep) / 4), rtol=1e-12)
    for bad in (0, 3, -2):
        with pytest.raises(E.EchoError):
            E.rotary_frequencies(bad)


def test_turns_of_a_frequency(tmp_path):
    """The fixed-point frequencies against exact fractions, compiled from the source by itself."""
    from fractions import Fraction

    sympy = pytest.importorskip("sympy")
    text = open(os.path.join(B.CSRC, "echo_ops_rotary.cu")).read()
    body = re.search(r"uint64_t rotary_turns\(double f\) \{.*?\n\}\n", text, re.S).group(0)
    f = [1.0, 0.1, 1e-4, 3.7, -0.3, 0.0, 2.0 ** 32, 1e-300, 6.283185307179586, 1 / 3]
    src = tmp_path / "turns.cpp"
    src.write_text("#include <cmath>\n#include <cstdint>\n#include <cstdio>\n" + body + "int main() { const double f[] = {" +
                   ", ".join(float(x).hex() for x in f) + "}; for (double x : f) printf(\"%llu\\n\", (unsigned long long)rotary_turns(x)); }\n")
    exe = str(tmp_path / "turns")
    subprocess.run(["g++", "-std=c++17", "-ffp-contract=off", str(src), "-o", exe], check=True)
    got = [int(s) for s in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    turn = Fraction(str(sympy.N(1 / (2 * sympy.pi), 90)))
    for x, g in zip(f, got):
        exact = Fraction(x) * turn * 2 ** 64
        off = (Fraction(g) - exact) % 2 ** 64
        off = min(off, 2 ** 64 - off)
        # f * high is exact with its rest; f * low and the sum are rounded: 2^-53 of f 2^-55, and the last bit
        assert off <= 2 + abs(x) * 2.0 ** (64 - 55 - 52), (x, float(off))
