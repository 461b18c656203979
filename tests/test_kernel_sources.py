"""What the kernels' sources state, held against what they contain."""
import os
import re

import numpy as np

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_02780_amd", "csrc")


def read(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def test_assembly_names_the_registers_that_it_writes():
    """A fixed register that an asm statement writes is in its list of clobbers, or the
    compiler may keep a value of its own there."""
    found = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith(".hip"):
            continue
        for text in re.findall(r"\basm(?:\s+volatile)?\s*\((.*?)\);", read(name), re.S):
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.split(":")[0]))
            for reg in re.findall(r"\b(?:s|v)_mov_b(?:32|64)\s+(m0|vcc|exec|[sv]\d+)\b", code):
                found += 1
                assert f'"{reg}"' in text.split(":")[-1], (name, reg, text)
    assert found > 0


def numbers(text):
    return [float(x) for x in re.findall(r"-?\d+(?:\.\d+)?(?:e-?\d+)?", text)]


def test_cap_approximations_keep_their_stated_errors():
    """The errors that the comments state for tanh(z) / z, against the constants evaluated in
    64 bits."""
    api, kernels = read("ss_api.cpp"), read("ss_attend.hip")
    comment = re.search(r"// v\[i\] <- cap tanh.*?\ntemplate", kernels, re.S).group(0)
    near, far = (float(x) for x in re.findall(r"2\^-(\d+\.\d+)", comment))
    near_to, far_to = (float(x) for x in re.findall(r"below (\d\.\d+)", comment))
    for name, bits, to in (("near_fit", near, near_to), ("fit", far, far_to)):
        c = numbers(re.search(r"double %s\[\d\] = \{(.*?)\}" % name, api).group(1))
        z = np.linspace(1e-6, to, 200001)
        err = np.abs(np.polynomial.polynomial.polyval(z * z, c) - np.tanh(z) / z)
        assert err.max() < 2.0 ** -bits, (name, float(np.log2(err.max())))
        assert err.max() > 2.0 ** -(bits + 0.2), (name, float(np.log2(err.max())))   # and not far more than it is
    # the continued fraction x / (1 + x^2 / (3 + ... )), cut where the comment says
    text = re.search(r"// tanh through exp.*?\n}", kernels, re.S).group(0)
    last, bits = int(re.search(r"cut after (\d+)", text).group(1)), float(re.search(r"less than 2\^-(\d+)", text).group(1))
    x = np.linspace(1e-6, 1.0, 200001)
    y, f = x * x, np.full(x.shape, float(last))
    for k in range(last - 2, 0, -2):
        f = k + y / f
    p, q = (np.array(numbers(re.search(r"float %s = (.*?);" % n, text).group(1).replace(".0f", ""))) for n in "pq")
    # p: fmaf(y, fmaf(y, a, b), c); q: fmaf(y, fmaf(y, y + a, b), c)
    num, den = (p[0] * y + p[1]) * y + p[2], ((y + q[0]) * y + q[1]) * y + q[2]
    assert np.abs(num / den * f - 1).max() < 1e-13
    assert np.abs(x / f - np.tanh(x)).max() < 2.0 ** -bits
