"""Warps that meet at a named barrier of their own (bar.sync with a count), which has no limit, go there together: a
bounded wait before it gives the same answer in all of them (mbar_wait_group), or a warp whose limit ran out would leave
and the others would wait for it without end. Read from the sources: that hang is not for a GPU to show."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_13660_gb300", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))
MEETS = re.compile(r"bar(?:rier)?(?:\.cta)?\.sync(?:\.aligned)?\s+[^;\"]*,")


def _code(path):
    with open(path) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def _first_unsafe(code):
    """The first meeting whose last wait before it, as the code is written, is a warp's own."""
    wrapper = re.search(r"void (\w+)\([^)]*\)\s*\{[^}]*" + MEETS.pattern, code)
    if not wrapper:
        return None
    body = code[wrapper.end():]
    last = None
    for m in re.finditer(rf"\b(mbar_wait\w*|{wrapper.group(1)})\(", body):
        if m.group(1).startswith("mbar_wait"):
            last = m.group(1)
        elif last not in (None, "mbar_wait_group"):
            return body[max(0, m.start() - 200):m.end()]
    return None


@pytest.mark.parametrize("path", FILES, ids=os.path.basename)
def test_a_group_waits_as_one(path):
    assert _first_unsafe(_code(path)) is None


def test_the_rule_sees_what_it_is_for():
    alone = "void meet(int g) { asm volatile(\"bar.sync %0, 128;\" ::\"r\"(g)); } if (!mbar_wait(&b, 0)) break; meet(1);"
    assert _first_unsafe(alone) and not _first_unsafe(alone.replace("mbar_wait(", "mbar_wait_group("))
    assert MEETS.search(_code(os.path.join(CSRC, "matmul.cu")))
