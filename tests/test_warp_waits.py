"""A role of a kernel that a whole warp walks through (one lane issues, chosen by elect_one) may not branch on what each lane has seen by itself: lanes that part there wait for one another for
good at the next elect, shuffle or vote.  The case in which they differ, a bounded wait that runs out in the moment in which its barrier completes, cannot be made on purpose; this looks at the sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1802_00130_b200", "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")))


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def roles(text):
    """(first line, body) of the branches of a kernel's warps: `if (warp == 0) {` to its end, and so on."""
    for m in re.finditer(r"if \(warp == \d\) \{|else \{", text):
        depth, j = 0, m.end() - 1
        while True:
            depth += {"{": 1, "}": -1}.get(text[j], 0)
            if depth == 0:
                break
            j += 1
        yield m.group(0), text[m.end():j]


def waits(body):
    """Each bounded wait: its line up to the call."""
    for m in re.finditer(r"\b(?:warp_)?wait_or_abort\(", body):
        yield body[body.rfind("\n", 0, m.start()) + 1:m.end()]


@pytest.mark.parametrize("name", FILES)
def test_waits_of_whole_warps_have_one_outcome(name):
    text = source(name)
    for first, body in roles(text):
        if "elect_one()" not in body or name == "tc_common.cuh":
            continue
        for line in waits(body):
            assert "warp_wait_or_abort(" in line or "lane == 0" in line, (name, first, line)


def test_the_outcome_is_a_vote():
    text = source("tc_common.cuh")
    at = text.index("bool warp_wait_or_abort(")
    assert "return __all_sync(0xffffffffu, wait_or_abort(" in text[at:text.index("}", at)]


def test_the_kernels_are_seen():
    """Those with such roles, and what the waits of others are: of one lane, or handed on by a shuffle."""
    elected = {f for f in FILES if "elect_one()" in source(f)} - {"tc_common.cuh"}
    assert elected == {f for f in FILES if "warp_wait_or_abort(" in source(f)} - {"tc_common.cuh"} and len(elected) >= 2
    for f in elected:
        assert sum("elect_one()" in body for _, body in roles(source(f))) >= 2
