"""A NaN among a row's logits, or among the teacher's logits in its slots, is one in the loss and in the whole of the row's
gradient, wherever it stands and whatever else the row holds; rows beside it, empty slots and rows of weight 0 are
left alone."""
import math

import pytest

from tests import _tokens as N

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("bucket", [False, True])
@pytest.mark.parametrize("cols", [40, 503, 12_001, 300_003])
@pytest.mark.parametrize("inplace", [False, True])
def test_the_whole_row(kind, bucket, cols, inplace):
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    n, K = 8, 6
    z = torch.randn(n, cols, device="cuda", generator=g).to(N.TYPES[kind])
    top, ids = torch.topk(z.float() + torch.randn(n, cols, device="cuda", generator=g), K, dim=1)
    lse = torch.logsumexp(torch.cat([top, top[:, :1] - 1], 1), 1) if bucket else None
    outside = torch.ones(n, cols, dtype=torch.bool, device="cuda").scatter_(1, ids, False)
    top[1, 2] = NAN                                     # the teacher's
    z[2, ids[2, 3]] = NAN                               # the student's, in a slot
    z[3, int(outside[3].nonzero()[cols // 2])] = NAN    # ... and in none
    z[4, outside[4]] = -INF                             # nothing outside of the slots, a NaN in one
    z[4, ids[4, 1]] = NAN
    z[5, outside[5]] = -INF
    top[5, 0] = NAN
    top[6, 1] = NAN                                     # weight 0
    ids[7, 5], top[7, 5] = -1, NAN                      # an empty slot
    weight = torch.tensor([1.0, 1.0, 2.0, -1.0, 1.0, 0.5, 0.0, 1.0], device="cuda")
    loss, d = torch.zeros(n, device="cuda"), z if inplace else torch.zeros_like(z)
    tok = pdb.pdb_tokens_create()
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, weight=weight, dlogits=d)
    assert torch.isnan(loss).tolist() == [False, True, True, True, True, True, True, False]
    assert torch.isnan(d[1:6]).all(1).tolist() == [True] * 5
    assert torch.isfinite(d[[0, 7]]).all() and torch.count_nonzero(d[6]) == 0
    pdb.check_tokens(tok)
