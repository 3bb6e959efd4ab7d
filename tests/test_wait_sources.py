"""Waits of the device code, checked on the sources: what one that is written wrongly does is not defined, so nothing that it
happens to do shows it."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_11101_b200", "csrc")
FILES = sorted(f for pattern in ("*.cu", "*.cuh") for f in glob.glob(os.path.join(CSRC, pattern)))


def _asm(text):
    """The strings of every asm statement, put together."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"\basm\b(?:\s+volatile)?\s*\(", text):
        yield "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text[m.end():text.index(";\n", m.end())].split("\n:")[0]))


def uniform_branches_on_waits(text):
    """asm statements that promise a branch to go one way for the whole warp (.uni) beside a try_wait, whose answer may differ from
    lane to lane."""
    return [code for code in _asm(text) if "try_wait" in code and re.search(r"\bbra\.uni\b", code)]


def test_the_check_sees_such_branches():
    good = 'asm volatile("{\\n.reg .pred p;\\nL:\\nmbarrier.try_wait.parity.shared::cta.b64 p, [%0], %1;\\n@p bra DONE;\\n}"\n: : "r"(a));\n'
    assert not uniform_branches_on_waits(good) and uniform_branches_on_waits(good.replace("bra DONE", "bra.uni DONE"))


@pytest.mark.parametrize("path", FILES, ids=[os.path.basename(f) for f in FILES])
def test_branches_on_a_wait_may_go_either_way(path):
    assert uniform_branches_on_waits(open(path).read()) == []
