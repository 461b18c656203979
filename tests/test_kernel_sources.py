"""What the kernels' sources state, held against what they contain."""
import os
import re

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
