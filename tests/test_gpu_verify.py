"""pdb_verify against the definition in 64 bits.  Tokens and counts are equal: the kernel decides drafts and draws on probabilities good to
2^-40, and the inputs' random numbers lie that close to a border with a probability below 1e-4 over all of these tests (a sum of V
terms has V borders, each 2^-40 wide).  Log probabilities are as near as those of pdb_logprobs."""
import math

import pytest

from tests._tokens import TYPES, U, Rows, assert_near

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create(0, 0)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(n, D, vocab, dtype, seed=0, masked=0.0, lookup=False, ragged=False, wide=False, scale=1.0):
    g = _gen(seed)
    z = torch.randn(n, D + 1, vocab, device="cuda", generator=g) * 2
    z += torch.where(torch.rand(z.shape, device="cuda", generator=g) < 4 / vocab, 9.0, 0.0)
    if masked:
        drop = torch.rand(z.shape, device="cuda", generator=g) < masked
        drop[..., vocab // 2] = False
        z.masked_fill_(drop, -math.inf)
    y = (z[:, :D] + 0.5 * torch.randn(n, D, vocab, device="cuda", generator=g)).to(dtype)
    z = z.to(dtype)
    if lookup:
        ids = torch.where(torch.rand(n, D, device="cuda", generator=g) < 0.7, z[:, :D].float().argmax(2),
                          torch.randint(0, vocab, (n, D), device="cuda", generator=g))
    else:
        q = torch.softmax(y.float() * scale, 2).view(n * D, vocab)
        ids = torch.multinomial(q, 1, generator=g).view(n, D) if n * D else torch.zeros(n, D, dtype=torch.int64, device="cuda")
    if ragged and D:
        ids = torch.where(torch.arange(D, device="cuda") < torch.randint(0, D + 1, (n, 1), device="cuda", generator=g), ids, -1)
    return (z.view(n * (D + 1), vocab), ids.to(torch.int64 if wide else torch.int32),
            torch.rand(n, D, device="cuda", generator=g), torch.rand(n, device="cuda", generator=g),
            None if lookup else y.view(n * D, vocab))


def _call(tok, z, ids, u, v, y, scale=1.0, draft_scale=1.0):
    n, D = ids.shape
    tokens = torch.full((n, D + 1), -7, device="cuda", dtype=torch.int32)
    accepted = torch.full((n,), -7, device="cuda", dtype=torch.int32)
    logp = torch.full((n, D + 1), math.nan, device="cuda")
    pdb.pdb_verify(tok, z, ids, u, v, tokens, accepted, draft=y, logp=logp, scale=scale, draft_scale=draft_scale)
    return tokens, accepted, logp


def _softmax(row, scale):
    x = row.double().cpu() * float(torch.tensor(scale, dtype=torch.float32))
    if torch.isnan(x).any() or (x == math.inf).any() or (x == -math.inf).all():
        return None
    e = (x - x.max()).exp()
    return e / e.sum()


def _want(z, ids, u, v, y, scale=1.0, draft_scale=1.0):
    n, D = ids.shape
    vocab = z.shape[1]
    tokens = torch.full((n, D + 1), -1, dtype=torch.int32)
    accepted = torch.zeros(n, dtype=torch.int32)
    for s in range(n):
        for d in range(D + 1):
            p = _softmax(z[s * (D + 1) + d], scale)
            t = int(ids[s, d]) if d < D else -1
            q = None
            if 0 <= t < vocab:
                q = torch.zeros(vocab, dtype=torch.float64).index_fill_(0, torch.tensor(t), 1.0) if y is None \
                    else _softmax(y[s * D + d], draft_scale)
            accepted[s] = d
            if p is None:
                break
            if q is not None and float(u[s, d]) * q[t] < p[t]:
                tokens[s, d] = t
                continue
            r = p if q is None else (p - q).clamp(min=0)
            if r.sum() == 0:
                r = p
            upto = r.cumsum(0)
            x = min(max(float(v[s]), 0.0), 1.0) if not math.isnan(float(v[s])) else 0.0
            j = int((upto <= x * upto[-1]).sum())
            tokens[s, d] = min(j, int(r.nonzero().max()))
            break
    return tokens, accepted


def _check(tok, z, ids, u, v, y, scale=1.0, draft_scale=1.0):
    tokens, accepted, logp = _call(tok, z, ids, u, v, y, scale, draft_scale)
    want, count = _want(z, ids, u, v, y, scale, draft_scale)
    assert torch.equal(accepted.cpu(), count)
    assert torch.equal(tokens.cpu(), want)
    R = Rows(z, scale)
    n, D = ids.shape
    at = want.clamp(min=0).long().view(-1, 1)
    there = want.view(-1) >= 0
    assert_near(logp.view(-1), torch.where(there, R.logp.gather(1, at)[:, 0], 0.0),
                torch.where(there, R.tol_logp.gather(1, at)[:, 0], 0.0), "logp")
    return tokens, accepted, logp


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,D,vocab", [(1, 0, 1), (1, 1, 2), (3, 2, 7), (2, 8, 255), (5, 3, 256), (4, 1, 257), (40, 4, 1000),
                                       (160, 2, 4099), (7, 5, 50_001), (1, 4, 128_000)])
@pytest.mark.parametrize("lookup", [False, True])
def test_tokens(tok, kind, n, D, vocab, lookup):
    _check(tok, *_inputs(n, D, vocab, TYPES[kind], seed=vocab + n, lookup=lookup))
    pdb.check_tokens(tok)


@pytest.mark.parametrize("masked,ragged,wide,scale,draft_scale", [(0.5, False, False, 1.0, 1.0), (0.99, True, True, 1.0, 1.0),
                                                                  (0.0, True, False, 1 / 0.7, 1 / 0.7), (0.0, False, True, 0.3, 2.0),
                                                                  (0.5, True, False, 40.0, 1e-3)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_masks_and_scales(tok, kind, masked, ragged, wide, scale, draft_scale):
    _check(tok, *_inputs(24, 4, 3001, TYPES[kind], seed=5, masked=masked, ragged=ragged, wide=wide, scale=draft_scale),
           scale, draft_scale)


def test_plain_draws(tok):
    # no drafts at all: a token for each row, all of a long row's places
    z, ids, u, _, y = _inputs(300, 0, 9001, torch.float32, seed=3)
    v = (torch.arange(300, device="cuda") + 0.5) / 300
    z = z[:1].expand(300, -1).contiguous()
    tokens, accepted, _ = _check(tok, z, ids, u, v, None)
    assert (tokens[1:] >= tokens[:-1]).all() and (accepted == 0).all()


@pytest.mark.parametrize("kind", list(TYPES))
def test_strides(tok, kind):
    z, ids, u, v, y = _inputs(6, 3, 1237, TYPES[kind], seed=9)
    for pad, first in ((5, 0), (8, 8), (3, 1)):
        wide = torch.full((z.shape[0], z.shape[1] + pad + first), math.nan, device="cuda", dtype=z.dtype)
        zs = wide[:, first:first + z.shape[1]]
        zs.copy_(z)
        ws = torch.full((y.shape[0], y.shape[1] + pad + 2 * first), math.inf, device="cuda", dtype=z.dtype)
        ys = ws[:, 2 * first:2 * first + z.shape[1]]
        ys.copy_(y)
        wi = torch.full((6, 5), -1, device="cuda", dtype=ids.dtype)
        wi[:, 1:4] = ids
        got, want = _call(tok, zs, wi[:, 1:4], u, v, ys), _call(tok, z, ids, u, v, y)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", list(TYPES))
def test_alone_and_among_others(tok, kind):
    # how many blocks a row is split over does not show in the tokens
    z, ids, u, v, y = _inputs(1, 4, 20_011, TYPES[kind], seed=21)
    one = _call(tok, z, ids, u, v, y)
    for n in (30, 200):
        many = _call(tok, z.repeat(n, 1), ids.repeat(n, 1), u.repeat(n, 1), v.repeat(n), y.repeat(n, 1))
        assert (many[0] == one[0]).all() and (many[1] == one[1]).all()


def test_equal_rows_are_accepted(tok):
    # p = q: u < 1 accepts, however near 1
    z, ids, _, v, _ = _inputs(50, 3, 5003, torch.bfloat16, seed=2)
    y = z.view(50, 4, -1)[:, :3].reshape(150, -1).contiguous()
    u = torch.full((50, 3), 1.0 - 2.0 ** -24, device="cuda")
    _, accepted, _ = _check(tok, z, ids, u, v, y)
    assert (accepted == 3).all()


@pytest.mark.parametrize("vocab", [8, 256, 4096])
def test_borders(tok, vocab):
    # equal logits: p = 1/V, sums of which are exact; u = p is not below p, and v V a whole number means that token
    z = torch.zeros(6, vocab, device="cuda")
    ids = torch.tensor([[1], [1], [1]], device="cuda")
    u = torch.tensor([[1 / vocab], [1 / vocab * (1 - 2.0 ** -24)], [0.0]], device="cuda")
    v = torch.tensor([0.0, 0.5, 0.75], device="cuda")
    tokens, accepted, _ = _call(tok, z, ids, u, v, None)
    assert accepted.tolist() == [0, 1, 1]
    assert tokens.tolist() == [[0, -1], [1, vocab // 2], [1, 3 * vocab // 4]]


@pytest.mark.parametrize("u,v", [(0.0, 0.0), (1.0 - 2.0 ** -24, 1.0 - 2.0 ** -24), (2.0 ** -40, 2.0 ** -30), (2.0 ** -140, 2.0 ** -149),
                                 (1.0, 1.0), (5.0, 7.0), (0.5, -1.0), (math.nan, math.nan)])
def test_ends_of_the_numbers(tok, u, v):
    z, ids, a, b, y = _inputs(9, 2, 777, torch.float32, seed=4, masked=0.3)
    a.fill_(u)
    b.fill_(v)
    _check(tok, z, ids, a, b, y)


@pytest.mark.parametrize("size", [1e-35, 1e-31, 1e-25, 1e25, 1e31, 1e35])
def test_far_scales(tok, size):
    # logits of any size and the scale that makes them ordinary ones
    z, ids, u, v, y = _inputs(30, 2, 2000, torch.float32, seed=17)
    _check(tok, z / size, ids, u, v, y / size, size, size)


@pytest.mark.parametrize("offset", [300.0, -3000.0, 1e6])
def test_far_offsets(tok, offset):
    # a distance that all logits share, which their type rounds
    z, ids, u, v, y = _inputs(30, 2, 2000, torch.float32, seed=18)
    _check(tok, z + offset, ids, u, v, y - offset)


def test_rows_without_a_distribution(tok):
    for bad in (math.nan, math.inf, -math.inf):
        for where in range(3):
            z, ids, u, v, y = _inputs(5, 2, 3000, torch.float32, seed=8)
            u.fill_(0.0)                                          # accepts what has a probability
            row = z.view(5, 3, -1)[2, where]
            if bad == -math.inf:
                row.fill_(bad)
            else:
                row[1777] = bad
            tokens, accepted, logp = _call(tok, z, ids, u, v, y)
            want, count = _want(z, ids, u, v, y)
            assert torch.equal(tokens.cpu(), want) and torch.equal(accepted.cpu(), count)
            assert accepted[2] == where and tokens[2, where] == -1 and not logp.isnan().any()
            if where < 2:                                         # a draft row without one ends the drafts
                z, ids, u, v, y = _inputs(5, 2, 3000, torch.float32, seed=8)
                u.fill_(0.0)
                row = y.view(5, 2, -1)[2, where]
                if bad == -math.inf:
                    row.fill_(bad)
                else:
                    row[1777] = bad
                tokens, accepted, logp = _check(tok, z, ids, u, v, y)
                assert accepted[2] == where and tokens[2, where] >= 0


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("scale", [1.0, 2.0, 0.25])
def test_masked_by_the_lowest_value(tok, kind, scale):
    low = torch.finfo(TYPES[kind]).min
    z, ids, u, v, y = _inputs(12, 2, 1500, TYPES[kind], seed=6)
    z[:, 100:1400] = low
    y[:, 50:1450] = low
    z[3] = low                                                    # a row masked from end to end is uniform
    ids[:, 1] = 700                                               # a drafted token that the target's mask leaves out
    _check(tok, z, ids, u, v, y, scale, scale)


def test_what_the_draft_alone_has(tok):
    # p lies inside q's mask: a refusal draws from the rest, which is p where q has nothing
    z = torch.full((2, 1000), -math.inf, device="cuda")
    z[:, 10] = z[:, 20] = 0.0
    y = torch.full((1, 1000), -math.inf, device="cuda")
    y[:, 20] = y[:, 30] = 0.0
    ids = torch.tensor([[30]], device="cuda", dtype=torch.int32)
    tokens, accepted, _ = _call(tok, z, ids, torch.zeros(1, 1, device="cuda"), torch.tensor([0.9], device="cuda"), y)
    assert accepted.tolist() == [0] and tokens.tolist() == [[10, -1]]


def test_ids_out_of_range(tok):
    mine = pdb.pdb_tokens_create(0, 0)
    z, ids, u, v, y = _inputs(6, 3, 500, torch.float32, seed=12)
    u.fill_(0.0)
    ids[1, 1], ids[2, 0], ids[4, 2] = 500, 1 << 30, -5
    _check(mine, z, ids, u, v, y)
    assert pdb.pdb_tokens_status(mine) == pdb.PDB_ERANGE


def test_optional_outputs(tok):
    z, ids, u, v, y = _inputs(6, 3, 500, torch.float32, seed=13)
    tokens = torch.empty(6, 4, device="cuda", dtype=torch.int32)
    pdb.pdb_verify(tok, z, ids, u, v, tokens, draft=y)
    assert torch.equal(tokens, _call(tok, z, ids, u, v, y)[0])


def test_largest_vocabulary(tok):
    z, ids, u, v, y = _inputs(2, 1, 1 << 21, torch.bfloat16, seed=14)
    _check(tok, z, ids, u, v, y)


def test_flat_long_rows(tok):
    # every token as probable as the next: the finest steps that a row of this length has
    g = _gen(3)
    z = (torch.randn(64, 200_003, device="cuda", generator=g) * 0.01)
    _check(tok, z, torch.zeros(64, 0, device="cuda", dtype=torch.int32), torch.zeros(64, 0, device="cuda"),
           torch.rand(64, device="cuda", generator=g), None)


def test_graphs_and_streams(tok):
    z, ids, u, v, y = _inputs(8, 3, 5000, torch.bfloat16, seed=30)
    want = _call(tok, z, ids, u, v, y)
    tokens, accepted, logp = (torch.empty_like(x) for x in want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pdb.pdb_verify(tok, z, ids, u, v, tokens, accepted, draft=y, logp=logp)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((tokens, accepted, logp), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pdb.pdb_verify(tok, z, ids, u, v, tokens, accepted, draft=y, logp=logp)
    z2, ids2, u2, v2, y2 = _inputs(8, 3, 5000, torch.bfloat16, seed=31)
    want = _call(tok, z2, ids2, u2, v2, y2)
    for a, b in ((z, z2), (ids, ids2), (u, u2), (v, v2), (y, y2)):
        a.copy_(b)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((tokens, accepted, logp), want))


def test_refusals(tok):
    z, ids, u, v, y = _inputs(2, 2, 50, torch.float32)
    tokens = torch.empty(2, 3, device="cuda", dtype=torch.int32)
    for kw in (dict(target=z[:5]), dict(draft_ids=ids.view(-1)), dict(draft_ids=ids.float()), dict(accept_u=u[:1]),
               dict(accept_u=u.double()), dict(draw_u=v.cpu()), dict(tokens=tokens.long()), dict(tokens=tokens[:, :2]),
               dict(draft=y.half()), dict(draft=y[:3]), dict(draft=y[:, :49]), dict(scale=0.0), dict(logp=torch.empty(2, 2, device="cuda"))):
        args = dict(target=z, draft_ids=ids, accept_u=u, draw_u=v, tokens=tokens, draft=y)
        args.update(kw)
        with pytest.raises(pdb.PdbError):
            pdb.pdb_verify(tok, **args)


def _wide_softmax(row, scale):
    np = pytest.importorskip("numpy")
    x = row.double().cpu().numpy().astype(np.longdouble) * np.longdouble(float(torch.tensor(scale, dtype=torch.float32)))
    e = np.exp(x - x.max())
    return e / e.sum()


def _close_calls(weights, n, seed):
    """n numbers in fp32 that lie 2^-36 to 2^-28 of the rows' sums from a border of the weights' running ones, and the tokens that they mean.  (The
    kernel's last resort rounds each of V weights to 2^-46 of the rows' sums: V^0.5 2^-47.8 together, 8 times that for V = 128,000 is 2^-36.3;
    of what p - q comes to it is more, by 1 / sum(p - q).)"""
    import numpy as np
    upto = np.cumsum(weights)
    border = upto / upto[-1]
    v = border.astype(np.float32)
    off = np.abs(v.astype(np.longdouble) - border) * upto[-1]
    where = np.nonzero((off > 2.0 ** -36) & (off < 2.0 ** -28) & (v > 0) & (v < 1) & (weights > 0))[0]
    # as many of each size
    size = np.floor(np.log2(off[where].astype(np.float64))).astype(int)
    r = np.random.default_rng(seed)
    chosen = np.concatenate([r.permutation(where[size == e])[:-(-n // 8)] for e in range(-36, -28)])[:n]
    v = v[chosen]
    return torch.from_numpy(v).cuda(), [int(np.sum(border <= np.longdouble(x))) for x in v]


@pytest.mark.parametrize("vocab,kind,scale", [(128_000, "bf16", 1.0), (128_000, "f32", 0.7), (32_001, "f16", 1.0), (50_000, "f32", 2.0), (128_000, "bf16", 0.01)])
@pytest.mark.parametrize("few", [False, True])
def test_numbers_close_to_borders(tok, vocab, kind, scale, few):
    # where the draw's margin decides: from p, from p - q, and from p without a token
    dtype = TYPES[kind]
    z = (torch.randn(1, vocab, device="cuda", generator=_gen(vocab)) * 2).to(dtype)
    y = (z.float() + 0.3 * torch.randn(1, vocab, device="cuda", generator=_gen(vocab + 1))).to(dtype)
    p, q = _wide_softmax(z[0], scale), _wide_softmax(y[0], scale)
    n, few_rows = 140, 20
    ran = 0
    for form in ("p", "p - q", "without"):
        t = int((q - p).argmax()) if form == "p - q" else int(p.argmin())
        w = p.copy()
        if form == "p - q":
            w = (p - q).clip(min=0)
        elif form == "without":
            w[t] = 0
        v, want = _close_calls(w, n, vocab)
        ran += len(want)
        D = 0 if form == "p" else 1
        for s0 in range(0, len(want), few_rows if few else n):
            part = v[s0:s0 + few_rows if few else None]
            m = part.numel()
            ids = torch.full((m, D), t, device="cuda", dtype=torch.int32)
            u = torch.ones(m, D, device="cuda")
            rows = z.expand(m * (D + 1), vocab).contiguous()
            tokens, accepted, _ = _call(tok, rows, ids, u, part, y.expand(m, vocab).contiguous() if form == "p - q" else None, scale, scale)
            assert (accepted == 0).all()
            assert tokens[:, 0].tolist() == want[s0:s0 + m], form
    assert ran >= 100


@pytest.mark.parametrize("vocab,kind,scale", [(128_000, "bf16", 1.0), (128_000, "f32", 0.7), (32_001, "f16", 1.0), (50_000, "f32", 2.0), (128_000, "bf16", 0.01)])
@pytest.mark.parametrize("few", [False, True])
def test_acceptances_close_to_equal(tok, vocab, kind, scale, few):
    # u q and p from 2^-12 to 2^-36 apart, by halves: from where the statistics decide to where the terms do, which are good to 2^-40.5 each
    import numpy as np
    dtype = TYPES[kind]
    z = (torch.randn(1, vocab, device="cuda", generator=_gen(vocab + 2)) * 2).to(dtype)
    y = (z.float() + 0.3 * torch.randn(1, vocab, device="cuda", generator=_gen(vocab + 3))).to(dtype)
    p, q = _wide_softmax(z[0], scale), _wide_softmax(y[0], scale)
    r = np.random.default_rng(vocab)
    tokens, numbers = [], []
    likely = np.nonzero(q > p)[0]
    for size in range(-36, -12):
        for sign in (-1, 1):
            t = r.choice(likely, 4000)
            u = (p[t] / q[t] * (1 + sign * 2.0 ** (size + 0.5))).astype(np.float32)
            off = u.astype(np.longdouble) * q[t] / p[t] - 1
            ok = np.nonzero((off * sign > 2.0 ** size) & (off * sign < 2.0 ** (size + 1)) & (u < 1))[0][:3]
            tokens += t[ok].tolist()
            numbers += u[ok].tolist()
    assert len(tokens) >= 100
    want = [float(np.longdouble(np.float32(u)) * q[t] - p[t]) < 0 for t, u in zip(tokens, numbers)]
    step = 20 if few else len(tokens)
    for s0 in range(0, len(tokens), step):
        part = tokens[s0:s0 + step]
        m = len(part)
        ids = torch.tensor(part, device="cuda", dtype=torch.int32).view(m, 1)
        u = torch.tensor(numbers[s0:s0 + step], device="cuda", dtype=torch.float32).view(m, 1)
        _, accepted, _ = _call(tok, z.expand(2 * m, vocab).contiguous(), ids, u, torch.full((m,), 0.5, device="cuda"), y.expand(m, vocab).contiguous(),
                               scale, scale)
        assert accepted.tolist() == [int(x) for x in want[s0:s0 + step]]
