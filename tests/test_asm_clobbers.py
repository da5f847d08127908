"""Inline assembly names every register that it writes behind the compiler's back."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_07177_amd", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "**", "*.h*"), recursive=True))


def statements(text):
    """The asm statements of a source: the assembly, and what stands behind the last colon."""
    for m in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[m.end():at - 1]


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_m0_is_named(path):
    with open(path) as f:
        for s in statements(f.read()):
            code = s.split(":")[0]
            if re.search(r"\bs_\w+\s+m0\b", code):
                assert '"m0"' in s.rsplit(":", 1)[1], s


def test_there_is_one_to_look_at():
    found = sum(bool(re.search(r"\bs_\w+\s+m0\b", s)) for p in FILES for s in statements(open(p).read()))
    assert found >= 1
