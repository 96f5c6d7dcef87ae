"""The token operators' kernels start while the kernel before them still runs, so each waits for that one's end before it
touches memory, and reads nothing by the loads for data that nobody writes while a kernel lives."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1508_00703_gb300", "csrc")
FILES = ["tokens.cuh", "rows.cuh", "embed.cu", "logprobs.cu", "distill.cu"]


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"/\*.*?\*/|//[^\n]*", "", text, flags=re.S)


@pytest.mark.parametrize("name", FILES)
def test_plain_loads(name):
    code = _code(name)
    assert "__ldg" not in code
    assert not re.search(r"\bld\.[\w.:]*\bnc\b", code)
    assert not re.search(r"\bconst\b[^,;(){}]*\*\s*(?:const\s*)?__restrict__", code)


@pytest.mark.parametrize("name", [f for f in FILES if f.endswith(".cu")])
def test_kernels_wait_first(name):
    code = _code(name)
    kernels = [m.start() for m in re.finditer(r"__global__", code)]
    assert kernels
    for at in kernels:
        body = code[code.index(")\n{", at) + 3:]
        before = body[:body.index("after_previous();")]
        lines = [x.strip() for x in before.split("\n") if x.strip()]
        assert all(re.fullmatch(r"(constexpr [^;]*;|using [^;]*;)", x) for x in lines), lines


def test_a_handle_does_not_hang_on_the_gradient_kernel():
    # what runs at once of pdb_distill's gradient is asked by that call: where a device has no room for its clusters, the other
    # operators work
    code = _code("embed.cu")
    body = code[code.index("int pdb_tokens_create"):code.index("int pdb_tokens_status")]
    assert "count_room" not in body and "Occupancy" not in body and "k_distill" not in code
