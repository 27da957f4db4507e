"""What test_read_only_loads.py asks of the kernels in .cu files, of those in headers and of the loads that headers' functions make for their callers."""
import os
import re

import pytest

from test_read_only_loads import CSRC, body, early_kernels, test_read_only_loads_go_through_dep as go_through_dep

HEADERS = sorted(f for f in os.listdir(CSRC) if f.endswith(".cuh"))
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh")))


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", HEADERS)
def test_kernels_in_headers(name):
    go_through_dep(name)


def test_a_kernel_in_a_header_is_seen():
    assert [k for f in HEADERS for k, _, _ in early_kernels(source(f))] == ["product4_kernel"]


def test_what_is_read_before_the_wait():
    """The products with 4-bit weights ask for weights, and look at the plan, before the wait where the call says that these are older than the kernel before: nothing else, and nowhere else.  The one
    call that says so is the layer's second product, whose first has waited for them."""
    text = source("weight4_product.cuh")
    kernel = body(text, text.index("product4_kernel(const"))
    before = kernel.split("grid_dep_wait();")[0]
    for m in re.finditer(r"\b(place|begin)\(\);|= (?:place|begin)\(\)", before):
        enclosing = before.rfind("if (p.early) {", 0, m.start())
        assert enclosing >= 0 and before[enclosing:m.start()].count("}") == 0, m.group(0)
    assert "p.x" not in before and "pair_of" not in before and "p.d" not in before
    early = [(f, line) for f in SOURCES for line in source(f).splitlines() if re.search(r"\bearly = true", line)]
    assert [f for f, _ in early] == ["weight4.cu"] and "b.early = true" in early[0][1] and "a.early" not in early[0][1]


@pytest.mark.parametrize("name", SOURCES)
def test_callers_hand_on_pointers_made_after_the_wait(name):
    """fetch_rows and fetch_chunk load through the read-only path what their callers name."""
    for line in source(name).splitlines():
        if re.search(r"\bfetch_(?:rows|chunk)\(", line) and "__device__" not in line and "const void* base" not in line:
            assert re.search(r"fetch_(?:rows|chunk)\(\w+, lane, (?:dep\(|base, ld)", line), line
