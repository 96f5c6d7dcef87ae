"""pdb_verify's acceptances where every rounding of the 32-bit statistics goes one way: a thread's sum stands at 16, and each of its 255 further chunks
adds a little less than half of its last digit, which is lost, or a little more, which counts twice.  That takes rows of 2^21 fp32
tokens that a block has to itself."""
import math

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

V, CHUNK = 1 << 21, 512 * 16


def _row(a, e):
    """One token of logit 0, a chunk's others at -a, and behind them 2^-24 (1 + e) of these."""
    z = torch.full((V,), -a - 24 * math.log(2) + math.log1p(e), device="cuda", dtype=torch.float32)
    z[:CHUNK] = -a
    z[5] = 0.0
    return z


@pytest.mark.parametrize("n", [3, 60])
def test_roundings_that_add_up(n):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    np = pytest.importorskip("numpy")
    tok = pdb.pdb_tokens_create(0, 0)
    # (a: what the rounding of a's exponential adds to the sums' errors is nearly the most that it can)
    zp, zq = _row(1.4048925638198853, -2.0 ** -10), _row(3.1798572540283203, 2.0 ** -10)
    p, q = (1 / np.exp(z.double().cpu().numpy().astype(np.longdouble)).sum() for z in (zp, zq))
    # u q from 2^-24 to 800 * 2^-24 above p and below it
    steps = np.concatenate([np.linspace(-800, 800, 241), np.linspace(480, 540, 60), np.linspace(-540, -480, 59)])
    u = (p / q * (1 + steps * 2.0 ** -24)).astype(np.float32)
    off = u.astype(np.longdouble) * q - p
    assert u.max() < 1 and (abs(off) > p * 2.0 ** -38).all()
    draft, target = zq.expand(n, V).contiguous(), zp.expand(2 * n, V).contiguous()
    got = []
    for s in range(0, len(u) if n == 60 else 2 * n, n):
        tokens = torch.empty(n, 2, device="cuda", dtype=torch.int32)
        accepted = torch.empty(n, device="cuda", dtype=torch.int32)
        pdb.pdb_verify(tok, target, torch.full((n, 1), 5, device="cuda", dtype=torch.int32), torch.from_numpy(u[s:s + n]).cuda().view(n, 1),
                       torch.full((n,), 0.5, device="cuda"), tokens, accepted, draft=draft)
        got += accepted.tolist()
    assert got == (off[:len(got)] < 0).astype(int).tolist()
