"""pdb_clip on a model's gradients in one flat buffer of more than 2^30 elements, which is one row, and on more than 2^31 rows: their number is limited
by 2^40 elements in all."""
import math

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

from tests.test_gpu_clip import REL, U  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [((1 << 30) + 9,), (1, (1 << 31) + 17), ((1 << 31) + 5, 1)])
def test_flat_buffers(shape):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    d = torch.full(shape, 2.0 ** -10, device="cuda", dtype=torch.bfloat16)
    n = d.numel()
    d.view(-1)[[5, n // 2, n - 1]] = 3.0
    norm = torch.empty(1, device="cuda")
    pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), 1.0, norm)
    N = math.sqrt((n - 3) * 2.0 ** -20 + 27)
    assert abs(float(norm) - N) <= (REL + U) * N
    # (neither value lies near a border between two of bfloat16's)
    low, high = (float(torch.tensor(x / N).bfloat16()) for x in (2.0 ** -10, 3.0))
    flat = d.view(-1)
    assert (flat[[5, n // 2, n - 1]].float() == high).all()
    flat[[5, n // 2, n - 1]] = low
    assert int((flat != low).sum()) == 0
