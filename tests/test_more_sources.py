"""The kernels of verify.cu, route.cu and clip.cu start while the kernel before them still runs: each waits for that one's end before it touches
memory, and reads nothing by the loads for data that nobody writes while a kernel lives."""
import pytest

from tests.test_tokens_sources import test_kernels_wait_first as waits_first
from tests.test_tokens_sources import test_plain_loads as plain_loads


@pytest.mark.parametrize("name", ["pack.cuh", "verify.cu", "route.cu", "clip.cu"])
def test_loads(name):
    plain_loads(name)


@pytest.mark.parametrize("name", ["verify.cu", "route.cu", "clip.cu"])
def test_waits(name):
    waits_first(name)
