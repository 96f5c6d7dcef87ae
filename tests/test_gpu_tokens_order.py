"""The order of pdb_embed_grad's sums, bit for bit: an id's rows in the order of the data, one after the other in pieces of 32,
and of a run over 32 every 8th piece together, then the eight sums in turn.  The values' sums depend on their order (sizes over
2^24, cancelling), so another order, or a sort that is not stable, gives other bits; that the values tell orders apart is
checked on the CPU for every case."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

PIECE, JOINED = 32, 8
# how often an id occurs: alone, about a piece, about the eight sums, many pieces
COUNTS = [1, 2, 3, 31, 32, 33, 63, 64, 65, 255, 256, 257, 288, 289, 513, 1000]


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


def _ids(n, vocab, rng):
    """n ids in any order, with the counts above in turn, one id for a tenth of them, and the rest by chance."""
    left, parts, names = n - n // 10, [np.full(n // 10, vocab - 1)], rng.permutation(vocab - 1)
    for i, name in enumerate(names[: vocab // 2]):
        c = COUNTS[i % len(COUNTS)]
        if c > left:
            break
        parts.append(np.full(c, name))
        left -= c
    parts.append(rng.choice(names[vocab // 2:], left))
    ids = np.concatenate(parts)
    return rng.permutation(ids)


def _values(n, dim, rng):
    size = np.exp2(rng.integers(-12, 13, (n, dim))).astype(np.float32)
    return (rng.standard_normal((n, dim)).astype(np.float32) * size).astype(np.float32)


def _run(rows, joined=JOINED):
    """Sum of one id's rows (count, dim) in the documented order, in fp32."""
    pieces = []
    for p in range(0, len(rows), PIECE):
        s = np.zeros(rows.shape[1], np.float32)
        for r in rows[p:p + PIECE]:
            s = s + r
        pieces.append(s)
    if len(pieces) == 1:
        return pieces[0]
    sums = []
    for w in range(min(joined, len(pieces))):
        s = np.zeros(rows.shape[1], np.float32)
        for piece in pieces[w::joined]:
            s = s + piece
        sums.append(s)
    total = np.zeros(rows.shape[1], np.float32)
    for s in sums:
        total = total + s
    return total


def _pairs(at):
    """Every two neighbours exchanged."""
    at = at.copy()
    even = len(at) // 2 * 2
    at[0:even:2], at[1:even:2] = at[1:even:2].copy(), at[0:even:2].copy()
    return at


def _tell(ids, d, vocab, scale, old, want):
    """Whether the values show other orders: the last first, neighbours exchanged, the pieces of a long run one after the other."""
    other = [_grad(ids, d, vocab, scale, old, lambda at: at[::-1]), _grad(ids, d, vocab, scale, old, _pairs)]
    if np.bincount(ids).max() > PIECE * JOINED:
        other.append(_grad(ids, d, vocab, scale, old, joined=1))
    return all((o != want).any() for o in other)


def _grad(ids, d, vocab, scale, old, order=lambda rows: rows, joined=JOINED):
    want = np.zeros((vocab, d.shape[1]), np.float32) if old is None else old.copy()
    by = np.argsort(ids, kind="stable")
    cuts = np.flatnonzero(np.diff(ids[by])) + 1
    for at in np.split(by, cuts):
        v = np.float32(scale) * _run(d[order(at)], joined)
        want[ids[at[0]]] = v if old is None else old[ids[at[0]]] + v
    return want


@pytest.mark.parametrize("n", [300, 2047, 2048, 2049, 8193, 20_000, 65_536, 65_537, 90_000])
@pytest.mark.parametrize("vocab,dim", [(40, 5), (700, 33), (5000, 8), (70_000, 64)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_order(n, vocab, dim, accumulate):
    rng = np.random.default_rng(n + dim)
    ids, d = _ids(n, vocab, rng), _values(n, dim, rng)
    old = _values(vocab, dim, rng) if accumulate else None
    want = _grad(ids, d, vocab, 0.3, old)
    assert _tell(ids, d, vocab, 0.3, old, want)
    tok = pdb.pdb_tokens_create(n, dim)
    table = torch.full((vocab, dim), 9.0, device="cuda") if old is None else torch.from_numpy(old.copy()).cuda()
    pdb.pdb_embed_grad(tok, torch.from_numpy(ids).cuda(), torch.from_numpy(d).cuda(), table, scale=0.3, accumulate=accumulate)
    assert np.array_equal(table.cpu().numpy(), want)
    pdb.check_tokens(tok)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
def test_order_of_16_bit_rows(kind):
    rng = np.random.default_rng(5)
    n, vocab, dim = 30_000, 3000, 136
    ids = _ids(n, vocab, rng)
    d = torch.from_numpy(_values(n, dim, rng)).to(kind)
    want = _grad(ids, d.float().numpy(), vocab, 1.0, None)
    assert _tell(ids, d.float().numpy(), vocab, 1.0, None, want)
    tok = pdb.pdb_tokens_create(n, dim)
    wide = torch.full((n, dim + 5), 3.0, device="cuda", dtype=kind)
    wide[:, 1:1 + dim] = d.cuda()
    for rows in (d.cuda(), wide[:, 1:1 + dim]):                  # wide moves, and element by element
        for out in (torch.float32, kind):
            grad = torch.empty(vocab, dim, device="cuda", dtype=out)
            pdb.pdb_embed_grad(tok, torch.from_numpy(ids).int().cuda(), rows, grad)
            assert torch.equal(grad.cpu(), torch.from_numpy(want).to(out))
