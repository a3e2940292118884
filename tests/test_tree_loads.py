"""Inline assembly that loads into LDS, held against what its instructions ask of each other: the compiler looks into no such block."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_31160_amd", "csrc")


def blocks():
    """(file, instructions, clobbers) of every block with a load into LDS."""
    got = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        with open(path) as f:
            text = f.read().replace("\\\n", "")
        for m in re.finditer(r"asm volatile\((.*?)\)\s*(?:;|\n)", text, re.S):
            body = m[1]
            code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', body.split("::")[0]))
            lines = [re.sub(r"\s+", " ", x).strip() for x in re.split(r"\\n|\\t|;", code)]
            lines = [x for x in lines if x]
            if any(x.startswith("buffer_load") and x.endswith("lds") for x in lines):
                got.append((os.path.basename(path), lines, re.findall(r'"(\w+)"', body.rsplit(":", 1)[1])))
    return got


def test_there_is_one():
    assert [name for name, _, _ in blocks()] == ["tree.hip"]


@pytest.mark.parametrize("block", blocks(), ids=lambda b: b[0])
def test_resource_registers_have_settled(block):
    """A scalar register that a vector instruction wrote is read by a vector load five wait states later at the earliest, and the
    instruction before the block may be such a write."""
    _, lines, _ = block
    waits = 0
    for x in lines:
        if x.startswith("buffer_load"):
            break
        waits += int(x.split()[1]) + 1 if x.startswith("s_nop") else 1
    assert waits >= 5


@pytest.mark.parametrize("block", blocks(), ids=lambda b: b[0])
def test_the_compiler_knows_what_is_overwritten(block):
    _, lines, clobbers = block
    assert any(x.startswith("s_mov_b32 m0") for x in lines) and "m0" in clobbers and "memory" in clobbers
