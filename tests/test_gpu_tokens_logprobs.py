"""pdb_logprobs and pdb_logprobs_grad against their formulas in 64 bits, with
bounds from fp32 rounding (tests/_tokens.py): vocabularies from one token to past
the longest split, rows at any alignment, masks down to nothing left, ties,
NaN and infinities, logits in any order, gradients by formula and difference."""
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


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lay(z, layout):
    """The same values as a tensor of its own, or as a view at an odd offset with a longer stride."""
    if layout == "whole":
        return z
    base = torch.full((z.shape[0], z.shape[1] + 5), 1e4, device="cuda").to(z.dtype)   # what lies between is large
    base[:, 3:3 + z.shape[1]] = z
    return base[:, 3:3 + z.shape[1]]


def _logits(n, cols, dtype, g, spread=3.0):
    return (torch.randn(n, cols, device="cuda", generator=g) * spread).to(dtype)


def _outputs(n, k):
    new = lambda *s: torch.full(s, 77.0, device="cuda")
    return dict(logp=new(n), lse=new(n), entropy=new(n), top_logp=new(n, k) if k else None,
                top_ids=torch.full((n, k), -7, device="cuda", dtype=torch.int32) if k else None)


def _check(tok, logits, ids, scale=1.0, k=0, ignore=-100):
    n, cols = logits.shape
    out = _outputs(n, k)
    pdb.pdb_logprobs(tok, logits, ids, scale=scale, ignore=ignore, **out)
    R = N.Rows(logits, scale)
    N.assert_near(out["lse"], R.lse, R.tol_lse, "lse")
    N.assert_near(out["entropy"], R.entropy, R.tol_entropy, "entropy")
    t = ids.long().cpu()
    there = (t >= 0) & (t < cols) & (t != ignore)
    at = torch.where(there, t, 0)[:, None]
    want = torch.where(there, R.logp.gather(1, at).squeeze(1), 0.0)
    want = torch.where(there & torch.isnan(R.lse), NAN, want)
    N.assert_near(out["logp"], want, torch.where(there, R.tol_logp.gather(1, at).squeeze(1), 0.0), "logp")
    if k:
        best = N.top(logits, k)
        assert torch.equal(out["top_ids"].cpu().long(), best)
        want = R.logp.gather(1, best)
        want = torch.where(torch.isnan(R.lse)[:, None], NAN, want)
        N.assert_near(out["top_logp"], want, R.tol_logp.gather(1, best), "top_logp")
    return out


COLS = [1, 2, 7, 8, 33, 255, 1000, 4099, 32_000, 50_001, 131_073]


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("cols", COLS)
def test_rows(tok, kind, cols):
    g = _gen(cols)
    for n, layout, k, scale in [(1, "whole", min(20, cols), 1.0), (3, "shifted", min(5, cols), 0.7),
                                (5, "whole", 0, 1.3)] + ([(700, "shifted", min(cols, 3), 1.0)] if cols < 1001 else []):
        z = _lay(_logits(n, cols, N.TYPES[kind], g), layout)
        ids = torch.randint(0, cols, (n,), device="cuda", generator=g)
        _check(tok, z, ids if n % 2 else ids.int().repeat_interleave(2)[::2], scale, k)
    pdb.check_tokens(tok)


@pytest.mark.parametrize("n,cols,k", [(2, 64, 64), (1, 300, 64), (9, 40_000, 64), (33, 2000, 33), (400, 128, 32),
                                      (150, 20_000, 1), (1, 200_000, 64), (2, 524_289, 7)])
def test_alternatives(tok, n, cols, k):
    g = _gen(n + k)
    ids = torch.randint(0, cols, (n,), device="cuda", generator=g)
    _check(tok, _logits(n, cols, torch.float32, g), ids, k=k)
    _check(tok, _logits(n, cols, torch.bfloat16, g), ids, k=k)                 # 8 bits of precision: many ties
    _check(tok, _logits(n, cols, torch.float16, g).round(), ids, k=k)          # a handful of values: ties everywhere


@pytest.mark.parametrize("cols", [64, 1000, 30_000])
@pytest.mark.parametrize("order", ["up", "down", "equal", "one-high", "block", "zeros-of-both-signs"])
def test_alternatives_in_any_order(tok, cols, order):
    up = torch.linspace(-5, 5, cols, device="cuda")
    z = {"up": up, "down": up.flip(0), "equal": torch.full_like(up, 2.0),
         "one-high": torch.where(torch.arange(cols, device="cuda") == cols - 1, 9.0, 0.0),
         # the large ones side by side, at an odd place
         "block": torch.where((torch.arange(cols, device="cuda") - cols // 3).abs() < 200, up + 20, up),
         "zeros-of-both-signs": torch.where(torch.arange(cols, device="cuda") % 3 == 0, -0.0, 0.0)}[order]
    z = torch.stack([z, z + 1, torch.roll(z, 1)])
    _check(tok, z, torch.tensor([0, cols - 1, cols // 2], device="cuda"), k=min(cols, 50))


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("cols", [9, 500, 40_000])
def test_masks(tok, kind, cols):
    g = _gen(11)
    dtype = N.TYPES[kind]
    lowest = torch.finfo(dtype).min
    z = _logits(8, cols, dtype, g)
    z[0, :] = -INF                                 # nothing left
    z[1, 1:] = -INF                                # one left
    z[2, torch.rand(cols, device="cuda", generator=g) < 0.9] = -INF
    z[2, 4] = 1.0
    z[3, 2:] = lowest                              # the type's lowest value: a mask that is not -inf
    z[4, :] = lowest                               # ... everywhere: uniform
    z[5, : cols - 2] = -INF
    z[6, ::2] = -INF
    ids = torch.tensor([3, 0, 4, 1, 5, cols - 1, 1, 2], device="cuda")
    _check(tok, z, ids, k=5)
    ids = torch.tensor([0, 5, 4, 6, 0, 0, 0, -100], device="cuda")             # given tokens that are masked out
    _check(tok, z, ids, k=min(cols, 50))
    pdb.check_tokens(tok)


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("cols", [10, 5000])
def test_nan_and_infinity(tok, kind, cols):
    g = _gen(12)
    z = _logits(5, cols, N.TYPES[kind], g)
    z[0, 3], z[1, cols - 1], z[2, 0], z[2, 7] = NAN, INF, NAN, NAN
    z[3, 1:] = -INF
    z[3, 5] = NAN
    out = _check(tok, z, torch.tensor([1, 2, 0, 4, 5], device="cuda"), k=4)
    assert torch.isfinite(out["logp"][4]) and torch.isnan(out["logp"][:4]).all()


def test_large_and_small_logits(tok):
    z = torch.tensor([[1e30, 1e30, -1e30, 0.0], [-3e38, -3e38, -3.1e38, -3e38], [80.0, -80.0, 0.0, 88.0],
                      [1e-40, 0.0, -1e-40, 2e-40], [3e38, -3e38, 0.0, 1.0]], device="cuda")
    _check(tok, z, torch.tensor([1, 0, 3, 3, 0], device="cuda"), k=2)


def test_ids_left_out_and_out_of_range():
    g = _gen(13)
    for whole, beyond in ((torch.int32, 500), (torch.int64, (1 << 32) + 3)):
        tok = pdb.pdb_tokens_create()
        z = _logits(4, 500, torch.float32, g)
        _check(tok, z, torch.tensor([1, -100, 2, -100], device="cuda", dtype=whole))
        _check(tok, z, torch.tensor([1, -1, 2, 3], device="cuda", dtype=whole), ignore=-1)
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_OK
        out = _check(tok, z, torch.tensor([1, beyond, 2, -1], device="cuda", dtype=whole))
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_ERANGE
        lse, H = out["lse"], out["entropy"]
        g1 = torch.ones(4, device="cuda")
        d = torch.full_like(z, 5.0)
        ids = torch.tensor([1, beyond, 2, -1], device="cuda", dtype=whole)
        pdb.pdb_logprobs_grad(tok, z, ids, lse, None, g1, None, d)
        assert torch.count_nonzero(d[1]) == 0 and torch.count_nonzero(d[3]) == 0
        want, tol = N.logprobs_grad(z, ids, 1.0, lse, None, g1, None, torch.float32)
        N.assert_near(d, want, tol, "dlogits")
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_ERANGE


def test_outputs_each_by_itself(tok):
    g = _gen(14)
    z = _logits(6, 3000, torch.bfloat16, g)
    ids = torch.randint(0, 3000, (6,), device="cuda", generator=g)
    whole = _check(tok, z, ids, k=8)
    for name in whole:
        alone = torch.zeros_like(whole[name])
        pdb.pdb_logprobs(tok, z, ids if name == "logp" else None, **{name: alone})
        assert torch.equal(alone, whole[name]), name
    some = {m: torch.zeros_like(whole[m]) for m in ("lse", "top_ids")}
    pdb.pdb_logprobs(tok, z, **some)
    assert all(torch.equal(some[m], whole[m]) for m in some)


def _grad(tok, z, ids, scale, g, h, layout="whole", inplace=False, lse=None, H=None):
    n = z.shape[0]
    out = _outputs(n, 0)
    pdb.pdb_logprobs(tok, z, ids, scale=scale, **{m: out[m] for m in ("logp", "lse", "entropy")})
    lse, H = out["lse"], out["entropy"]
    want, tol = N.logprobs_grad(z, ids, scale, lse, H, g, h, z.dtype)
    d = z if inplace else _lay(torch.full_like(z.contiguous(), 3.0), layout)
    pdb.pdb_logprobs_grad(tok, z, ids, lse, H, g, h, d, scale=scale)
    N.assert_near(d, want, tol, "dlogits")
    return d


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("cols", [1, 2, 7, 33, 1000, 4099, 50_001])
def test_gradient(tok, kind, cols):
    g = _gen(cols + 1)
    for n, zl, dl, scale in [(1, "whole", "whole", 1.0), (4, "shifted", "shifted", 0.7), (3, "whole", "shifted", 1.0),
                             (6, "shifted", "whole", 1.5)]:
        z = _lay(_logits(n, cols, N.TYPES[kind], g), zl)
        ids = torch.randint(0, cols, (n,), device="cuda", generator=g).int()
        a = torch.randn(n, device="cuda", generator=g)
        b = torch.randn(n, device="cuda", generator=g) * 0.1
        for x, y in ((a, b), (a, None), (None, b)):
            _grad(tok, z, ids, scale, x, y, dl)
    _grad(tok, _lay(_logits(5, cols, N.TYPES[kind], g), "shifted"), torch.zeros(5, device="cuda", dtype=torch.int64), 1.0,
          torch.randn(5, device="cuda", generator=g), torch.randn(5, device="cuda", generator=g), inplace=True)
    pdb.check_tokens(tok)


def test_gradient_of_masked_and_odd_rows(tok):
    g = _gen(16)
    z = _logits(7, 900, torch.float32, g)
    z[0] = -INF
    z[1, 5:] = -INF
    z[2, 3:] = torch.finfo(torch.float32).min
    z[3, 9] = NAN
    z[4, 9] = NAN
    z[5, :] = NAN
    ids = torch.tensor([1, 2, 0, 4, 4, 4, -100], device="cuda")
    a = torch.tensor([1.0, -2.0, 1.0, 1.0, 0.0, 0.0, 3.0], device="cuda")
    b = torch.tensor([0.5, 0.3, 0.2, 0.1, 0.0, 0.0, 0.0], device="cuda")
    d = _grad(tok, z, ids, 1.0, a, b)
    for r in (0, 4, 5, 6):                         # nothing left, or both coefficients zero
        assert torch.count_nonzero(d[r]) == 0
    assert torch.isnan(d[3]).all()


def test_gradient_against_differences(tok):
    # central differences of the formula in 64 bits; step h gives h^2 / 6 times the third derivative (< 1 for
    # these sums, whose coefficients are below 2) plus 64-bit rounding over h
    g = _gen(17)
    n, cols, step = 3, 11, 1e-4
    z = _logits(n, cols, torch.float32, g, 1.5)
    ids = torch.tensor([2, 10, 0], device="cuda")
    a, b = torch.tensor([1.0, -0.5, 2.0], device="cuda"), torch.tensor([0.3, 1.0, -0.7], device="cuda")
    d = _grad(tok, z, ids, 0.8, a, b).double().cpu()
    s = float(torch.tensor(0.8, dtype=torch.float32))

    def value(x):
        lp = torch.log_softmax(x * s, 1)
        H = -(lp.exp() * lp).sum(1)
        return (a.double().cpu() * lp[torch.arange(n), ids.cpu()] + b.double().cpu() * H).sum()
    x = z.double().cpu()
    _, tol = N.logprobs_grad(z, ids, 0.8, N.Rows(z, 0.8).lse.float(), N.Rows(z, 0.8).entropy.float(), a, b, torch.float32)
    for r in range(n):
        for j in range(cols):
            e = torch.zeros_like(x)
            e[r, j] = step
            diff = float((value(x + e) - value(x - e)) / (2 * step))
            # the kernel's own lse and entropy are rounded to fp32: 1e-6 of the coefficients covers it
            assert abs(diff - float(d[r, j])) <= float(tol[r, j]) + 8 * step ** 2 + 1e-10 + 1e-6 * 3


def test_rows_past_two_to_the_31_elements(tok):
    n, cols = 17_000, 131_072                      # 2.2e9 logits of 16 bits
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    z = torch.zeros(n, cols, dtype=torch.bfloat16, device="cuda")
    z[-1, 5], z[-2, cols - 1] = 20.0, 18.0
    ids = torch.full((n,), 5, device="cuda", dtype=torch.int32)
    out = _outputs(n, 2)
    pdb.pdb_logprobs(tok, z, ids, **out)
    R = N.Rows(z[-3:], 1.0)
    N.assert_near(out["logp"][-3:], R.logp[:, 5], R.tol_logp[:, 5], "logp")
    assert out["top_ids"][-3:].tolist() == [[0, 1], [cols - 1, 0], [5, 0]]
    one = torch.zeros(n, device="cuda")
    one[-3:] = 1.0
    pdb.pdb_logprobs_grad(tok, z, ids, out["lse"], None, one, None, z)
    want, tol = N.logprobs_grad(torch.zeros(1, cols), ids[-3:-2], 1.0, out["lse"][-3:-2], None, one[-3:-2], None, z.dtype)
    N.assert_near(z[-3:-2], want, tol, "dlogits")
    assert torch.count_nonzero(z[:-3]) == 0
    pdb.check_tokens(tok)


def test_same_bits_each_time_and_for_each_row_alone(tok):
    g = _gen(18)
    z = _logits(40, 9000, torch.bfloat16, g)
    ids = torch.randint(0, 9000, (40,), device="cuda", generator=g)
    a, b = _check(tok, z, ids, k=6), _check(tok, z, ids, k=6)
    assert all(torch.equal(a[m], b[m]) for m in a)


def test_on_another_stream(tok):
    side = torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    z = torch.zeros(3, 4000, device="cuda")
    torch.cuda.synchronize()
    own = pdb.pdb_tokens_create()
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-4
        z[:, 7] = 5.0
        out = _outputs(3, 1)
        pdb.pdb_logprobs(own, z, torch.full((3,), 7, device="cuda"), **out)
        d = torch.empty_like(z)
        pdb.pdb_logprobs_grad(own, z, torch.full((3,), 7, device="cuda"), out["lse"], None,
                              torch.ones(3, device="cuda"), None, d)
    side.synchronize()
    assert out["top_ids"].flatten().tolist() == [7, 7, 7]
    lse = math.log(3999 + math.exp(5.0))
    assert torch.allclose(out["logp"], torch.full((3,), 5.0 - lse, device="cuda"), atol=1e-5)
    assert torch.allclose(d[:, 7], torch.full((3,), 1 - math.exp(5.0 - lse), device="cuda"), atol=1e-5)


def test_refusals(tok):
    f = lambda *shape, **kw: torch.zeros(*shape, device="cuda", **kw)
    i = lambda n, dtype=torch.int32: torch.zeros(n, device="cuda", dtype=dtype)

    def refused(code, call, *a, **kw):
        with pytest.raises(pdb.PdbError) as e:
            call(*a, **kw)
        assert e.value.code == code, e.value
    z = f(4, 100)
    for a, kw in [((z, i(3)), dict(logp=f(3))), ((z, i(4)), dict(logp=f(3))), ((z, i(4)), {}), ((z,), dict(logp=f(4))),
                  ((z, f(4)), dict(logp=f(4))), ((z.double(), i(4)), dict(logp=f(4))), ((z.t(), i(100)), dict(logp=f(100))),
                  ((z, i(4)), dict(logp=f(4), lse=f(4).half())), ((z, i(4)), dict(logp=f(4), entropy=f(8)[::2])),
                  ((z,), dict(top_logp=f(4, 101))), ((z,), dict(top_logp=f(3, 5))), ((z,), dict(top_logp=f(5))),
                  ((z,), dict(top_logp=f(4, 5), top_ids=f(4, 5))), ((z,), dict(top_logp=f(4, 5), top_ids=f(4, 6).int())),
                  ((z,), dict(lse=f(4).cpu())), ((z,), dict(lse=f(4), scale=0.0)), ((z,), dict(lse=f(4), scale=-1.0)),
                  ((z,), dict(lse=f(4), scale=NAN)), ((f(4, 0),), dict(top_logp=f(4, 1)))]:
        refused(pdb.PDB_EINVAL, pdb.pdb_logprobs, tok, *a, **kw)
    refused(pdb.PDB_ETOOBIG, pdb.pdb_logprobs, tok, z, top_logp=f(4, 65))
    for a in [(z, i(4), f(4), f(4), f(4), f(4), f(4, 99)), (z, i(4), f(4), f(4), f(4), f(4), f(4, 100).half()),
              (z, i(4), None, f(4), f(4), f(4), f(4, 100)), (z, i(4), f(4), None, f(4), f(4), f(4, 100)),
              (z, None, f(4), f(4), f(4), f(4), f(4, 100)), (z, i(4), f(3), f(4), f(4), f(4), f(4, 100)),
              (z[:2], i(2), f(2), f(2), f(2), f(2), z[1:3])]:
        refused(pdb.PDB_EINVAL, pdb.pdb_logprobs_grad, tok, *a)


def test_without_columns(tok):
    lse, H = torch.ones(3, device="cuda"), torch.ones(3, device="cuda")
    pdb.pdb_logprobs(tok, torch.empty(3, 0, device="cuda"), lse=lse, entropy=H)
    assert lse.tolist() == [-INF] * 3 and H.tolist() == [0.0] * 3


@pytest.mark.parametrize("n,cols,k", [(1, 4470, 32), (8, 4372, 32), (3, 2051, 64), (20, 8200, 17), (245, 3728, 32), (2, 70_000, 64)])
def test_alternatives_of_short_shares(tok, n, cols, k):
    # few vectors for a block's threads, alone or split over a cluster; most of a row masked
    g = _gen(cols + k)
    ids = torch.randint(0, cols, (n,), device="cuda", generator=g)
    z = _logits(n, cols, torch.float16, g)
    _check(tok, z, ids, k=k)
    drop = torch.rand(n, cols, device="cuda", generator=g) < 0.97
    drop[:, -k:] = False
    _check(tok, _lay(z.float().masked_fill(drop, -INF), "shifted"), ids, k=k)
