"""pdb_logprobs_grad against the formula by differences from the row's maximum, in 64 bits, for logits whose size is far
above their differences: offsets of thousands and millions, rows masked by the type's lowest value from end to end, and
sums whose logarithm passes fp32's range once scaled.

The bound: with d = z - max and the terms of tests/_tokens.py, p is off by rel_p = (its row's sum) + U (2 |d| + |log p| + 8), and by
6 U |lse| where lse is below 256 and p is formed from it; the bracket's terms by a rounding each, the entropy by its own bound."""
import math

import pytest

from tests import _tokens as N

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

INF = math.inf
U, SLACK = N.U, N.SLACK


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create()


def _want(z, ids, scale, a, b):
    R = N.Rows(z, scale)
    s = float(torch.tensor(scale, dtype=torch.float32))
    n, cols = R.z.shape
    one = torch.zeros(n, cols, dtype=torch.float64)
    one[torch.arange(n), ids.long().cpu()] = 1.0
    g, h = a.double().cpu()[:, None], b.double().cpu()[:, None]
    H, lp = R.entropy[:, None], R.held
    want = s * (g * (one - R.p) - h * R.p * (lp + H))
    d = torch.where(R.p > 0, R.z - R.z.amax(1, keepdim=True), 0.0).abs()
    near = torch.where(R.lse.abs() < 256, R.lse.abs(), 0.0)
    rel_p = R.rel_s[:, None] + U * (2 * d + lp.abs() + 8 + 6 * near[:, None])
    tol = g.abs() * (R.p * rel_p + 3 * U * (one + R.p))
    tol = tol + h.abs() * R.p * ((lp.abs() + H.abs()) * (rel_p + 6 * U) + rel_p + R.tol_entropy[:, None])
    want = torch.where(R.none[:, None], 0.0, want)
    tol = SLACK * s * torch.where(R.none[:, None], 0.0, tol)
    return want, tol + N.rounding(want, z.dtype) + abs(s) * (g.abs() + h.abs() * 128) * 2.0 ** -126


def _check(tok, z, scale, seed, inplace):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, cols = z.shape
    ids = torch.randint(0, cols, (n,), device="cuda", generator=g)
    a, b = torch.randn(n, device="cuda", generator=g), torch.randn(n, device="cuda", generator=g) * 0.1
    out = {m: torch.empty(n, device="cuda") for m in ("logp", "lse", "entropy")}
    pdb.pdb_logprobs(tok, z, ids, scale=scale, **out)
    want, tol = _want(z, ids, scale, a, b)
    d = z if inplace else torch.full_like(z, 3.0)
    pdb.pdb_logprobs_grad(tok, z, ids, out["lse"], out["entropy"], a, b, d, scale=scale)
    N.assert_near(d, want, tol, "dlogits")
    return d


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("cols", [1, 9, 500, 4099, 50_001])
@pytest.mark.parametrize("scale", [1.0, 0.7, 2.0])
@pytest.mark.parametrize("inplace", [False, True])
def test_offsets(tok, kind, cols, scale, inplace):
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    dtype = N.TYPES[kind]
    shift = torch.tensor([0.0, 100.0, -250.0, 270.0, -300.0, 4000.0, -5000.0, 30_000.0, -60_000.0], device="cuda")
    if kind != "f16":
        shift = torch.cat([shift, torch.tensor([1e6, -3e7, 1e30, -3e38], device="cuda")])
    z = (torch.randn(len(shift), cols, device="cuda", generator=g) * 2 + shift[:, None]).to(dtype)
    z[2, ::3], z[6, ::3] = -INF, -INF                  # masked among them
    z[2, 0], z[6, 0] = shift[2], shift[6]
    _check(tok, z, scale, cols + 1, inplace)
    pdb.check_tokens(tok)


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("n,cols", [(4, 7), (4, 3001), (4, 128_000), (400, 2000)])
@pytest.mark.parametrize("scale", [1.0, 0.7, 1.7])
def test_rows_masked_from_end_to_end(tok, kind, n, cols, scale):
    # the type's lowest value everywhere: uniform, 1 / cols each; above a scale of 1 the logarithm of the sum is -inf in fp32
    dtype = N.TYPES[kind]
    z = torch.full((n, cols), torch.finfo(dtype).min, device="cuda", dtype=dtype)
    z[1] = -INF                                        # nothing left
    z[2] = torch.finfo(dtype).max
    z[3] = 0.0
    for inplace in (False, True):
        d = _check(tok, z.clone(), scale, n, inplace)
        assert torch.count_nonzero(d[1]) == 0


def test_many_rows_in_pieces_and_whole():
    # rows that are read as a whole beside rows that are not, each row written once
    own = pdb.pdb_tokens_create()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for n, cols in ((3, 200_000), (40, 60_001), (500, 9000)):
        z = torch.randn(n, cols, device="cuda", generator=g)
        z[::2] += 1e5
        _check(own, z.clone(), 1.0, 4, False)
        _check(own, z.clone(), 1.0, 4, True)
