"""Who issues the copies of cache blocks and queries (csrc): one thread of a warp, wherever one is issued.  Several threads
that issue together, each with its own operands, are what ended with an illegal address; this is seen by reading."""
import glob
import os
import re

import pytest

from conftest import ROOT

SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2608_02244_gb300", "csrc", "kv_*.cu")))
CALL = re.compile(r"\btma_load4?\(")
ONE = {"one", "(threadIdx.x & 127) == 0"}         # of a warp, or of a group of four


def guard(lines, at):
    """The condition of the nearest `if` at or above a line."""
    for i in range(at, -1, -1):
        m = re.search(r"\bif \((.*)", lines[i][:CALL.search(lines[i]).start()] if i == at else lines[i])
        if m:
            depth, text = 1, m.group(1)
            for k, c in enumerate(text):
                depth += (c == "(") - (c == ")")
                if depth == 0:
                    return text[:k]
    return None


def calls():
    for path in SOURCES:
        lines = open(path).read().split("\n")
        for at, line in enumerate(lines):
            if CALL.search(line.split("//")[0]):
                yield os.path.basename(path), lines, at


def test_all_kernels_with_copies_are_looked_at():
    assert {name for name, _, _ in calls()} == {"kv_attend.cu", "kv_prefix.cu", "kv_prompt.cu"}


@pytest.mark.parametrize("name,lines,at", [pytest.param(*c, id=f"{c[0]}:{c[2] + 1}") for c in calls()])
def test_one_thread_issues(name, lines, at):
    assert guard(lines, at) in ONE, lines[at]
