"""What lies behind a sequence's first refusal, or behind its last draft, changes nothing that pdb_verify gives, however many sequences there are:
of few the statistics of all rows are formed at once, of many a row's when its position is reached."""
import math

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

from tests.test_gpu_verify import _call, _inputs  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 5, 60, 90, 400])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf, 3e38])
@pytest.mark.parametrize("lookup", [False, True])
def test_rows_behind(n, kind, fill, lookup):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    D, vocab = 4, 2003
    tok = pdb.pdb_tokens_create(0, 0)
    z, ids, u, v, y = _inputs(n, D, vocab, kind, seed=n, lookup=lookup, ragged=True)
    want = _call(tok, z, ids, u, v, y)
    there = torch.arange(D + 1, device="cuda") <= want[1][:, None]          # positions that count
    z.view(n, D + 1, vocab)[~there] = fill
    if not lookup:
        y.view(n, D, vocab)[~there[:, :D]] = fill
        # (a position whose drafts have ended reads no draft row)
        y.view(n, D, vocab)[ids < 0] = fill
    u[~there[:, :D]] = math.nan
    ids[~there[:, :D] & (torch.arange(D, device="cuda") > want[1][:, None])] = -5
    got = _call(tok, z, ids, u, v, y)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    pdb.check_tokens(tok)
