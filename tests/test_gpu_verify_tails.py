"""pdb_verify's draws from rows with one large logit and a long tail of equal ones, whose roundings all go one way.  Tokens are equal to the definition's
in extended precision.  Terms are good to 2^-40 of themselves, so a border of the tail is known to 2^-40 of the tail from p (2^-23 of a token
of 128,000), and to 2^-40 of the rows' sums from p - q, whose head's two terms are subtracted: numbers that lie nearer to a
border than four times that are left out."""
import math

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

V = 128_000


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create(0, 0)


def _draw(tok, z, v, t=None, y=None):
    """The tokens drawn from row z with numbers v: from it alone, without token t, or from what it has more than row y."""
    n, D = v.numel(), 0 if t is None else 1
    ids = torch.full((n, D), -1 if t is None else t, device="cuda", dtype=torch.int32)
    tokens = torch.full((n, D + 1), -7, device="cuda", dtype=torch.int32)
    draft = None if y is None else y.expand(n, -1).contiguous()
    pdb.pdb_verify(tok, z.expand(n * (D + 1), -1).contiguous(), ids, torch.ones(n, D, device="cuda"), v, tokens, draft=draft)
    return tokens[:, 0].cpu()


def _weights(z):
    np = pytest.importorskip("numpy")
    x = z.double().cpu().numpy().astype(np.longdouble)
    return np.exp(x - x.max())


def _numbers(weights, near, n, seed):
    """n numbers whose places lie evenly over the tail, and the tokens that they mean."""
    import numpy as np
    upto = np.cumsum(weights)
    low = np.sort(weights[weights > 0])[:-1].sum()             # the tail
    start = upto[-1] - low if weights[0] > low else np.longdouble(0)
    r = np.random.default_rng(seed)
    places = start + low * r.random(4 * n).astype(np.longdouble)
    v = (places / upto[-1]).astype(np.float32)
    place = v.astype(np.longdouble) * upto[-1]
    j = np.searchsorted(upto, place, side="right")
    ok = (v < 1) & (j < weights.size)
    j = np.minimum(j, weights.size - 1)
    below = np.where(j > 0, upto[np.maximum(j - 1, 0)], np.longdouble(0))
    ok &= np.minimum(place - below, upto[j] - place) > near
    v, j = v[ok][:n], j[ok][:n]
    return torch.from_numpy(v).cuda(), torch.from_numpy(j.astype(np.int32))


def _row(gap, where, kind):
    z = torch.full((1, V), 3.0 - gap, device="cuda")
    z[0, where] = 3.0
    return z.to(kind)


# (behind the head, a number close to 1 still tells a tail of 2^-24 of it; before it, numbers close to 0 tell any)
PLACES = [(gap, where) for where in (0, 777, V - 1) for gap in (16.0, 18.0, 20.0, 22.0, 26.0)] + [(30.0, V - 1), (34.0, V - 1)]


@pytest.mark.parametrize("gap,where", PLACES)
@pytest.mark.parametrize("n", [12, 400])
def test_equal_tails(tok, gap, where, n):
    z = _row(gap, where, torch.float32)
    w = _weights(z[0])
    v, want = _numbers(w, 4 * 2.0 ** -40 * float(V * math.exp(-gap)), n, int(gap) + where)
    assert v.numel() >= min(n, 10)
    for s in range(0, v.numel(), n):
        assert torch.equal(_draw(tok, z, v[s:s + n]), want[s:s + n])
    # without one of the tail's tokens
    w = w.copy()
    w[5000] = 0
    v, want = _numbers(w, 4 * 2.0 ** -40 * float(V * math.exp(-gap)), n, int(gap) + where)
    assert torch.equal(_draw(tok, z, v, t=5000), want)


@pytest.mark.parametrize("gap", [14.0, 16.0, 18.0])
@pytest.mark.parametrize("n", [12, 400])
def test_equal_tails_of_differences(tok, gap, n):
    # the draft's head is lower and its tail too, but for every other token
    z, y = _row(gap, 0, torch.float32), _row(gap + 0.5, 0, torch.float32)
    y[:, 1::2] += 1.0
    y[:, V // 2] = 2.5
    p, q = _weights(z[0]), _weights(y[0])
    p, q = p / p.sum(), q / q.sum()
    w = (p - q).clip(min=0)
    assert w[0] > 0.3 and (w > 0).sum() > V // 3
    v, want = _numbers(w, 4 * 2.0 ** -40, n, int(gap))
    assert v.numel() >= min(n, 10)
    assert torch.equal(_draw(tok, z, v, t=V // 2, y=y), want)


@pytest.mark.parametrize("n", [1, 400])
def test_the_first_token_that_has_a_weight(tok, n):
    # v = 0 is the smallest token with any weight: 2^-90 of the largest is one
    z = torch.full((1, 5000), -math.inf, device="cuda")
    z[0, 40] = -60.0
    z[0, 70] = -30.0
    z[0, 4000] = 0.0
    v = torch.zeros(n, device="cuda")
    assert (_draw(tok, z, v) == 40).all()
    assert (_draw(tok, z, v, t=40) == 70).all()
    y = z.clone()
    y[0, 40] = -59.0
    y[0, 70] = -31.0
    assert (_draw(tok, z, v, t=4000, y=y) == 70).all()
