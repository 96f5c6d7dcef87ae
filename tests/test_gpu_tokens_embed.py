"""pdb_embed and pdb_embed_grad against their formulas in 64 bits.

The lookup is exact: one fp32 product, rounded once.  The gradient's bound is
that of an fp32 sum of the run's length (tests/_tokens.py).  Lengths from no id
to runs of tens of thousands, odd columns, rows at any alignment, ids in both
widths, ids that are left out, tables past 2^31 elements, other streams."""
import pytest

from tests import _tokens as N

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(rows, cols, dtype, g, layout="whole", scale=1.0):
    """rows x cols of normal values: a tensor of its own, or a view into a wider one at an odd offset."""
    if layout == "whole":
        return (torch.randn(rows, cols, device="cuda", generator=g) * scale).to(dtype)
    extra = {"shifted": 3, "padded": 8}[layout]
    base = (torch.randn(rows, cols + extra, device="cuda", generator=g) * scale).to(dtype)
    return base[:, 1:cols + 1] if layout == "shifted" else base[:, :cols]


def _zipf(n, vocab, g):
    w = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -1.0
    return torch.randperm(vocab, device="cuda", generator=g)[torch.multinomial(w, n, replacement=True, generator=g)]


@pytest.mark.parametrize("table_type", list(N.TYPES))
@pytest.mark.parametrize("out_type", list(N.TYPES))
@pytest.mark.parametrize("n,vocab,dim,layout", [(1, 1, 1, "whole"), (5, 3, 7, "shifted"), (33, 100, 8, "whole"),
                                               (1000, 50, 33, "padded"), (257, 1000, 1000, "shifted"),
                                               (64, 4000, 2050, "whole"), (3, 10, 4096, "padded"),
                                               (4099, 777, 64, "whole")])
def test_lookup_is_exact(table_type, out_type, n, vocab, dim, layout):
    g = _gen(1)
    table = _matrix(vocab, dim, N.TYPES[table_type], g, layout)
    out = _matrix(n, dim, N.TYPES[out_type], g, layout)
    tok = pdb.pdb_tokens_create()
    for whole in (torch.int32, torch.int64):
        ids = torch.randint(0, vocab, (n,), device="cuda", generator=g).to(whole)
        pdb.pdb_embed(tok, table, ids, out, scale=1.7)
        want = (table[ids.long()].float() * 1.7).to(out.dtype)
        assert torch.equal(out, want)
    pdb.check_tokens(tok)


def test_lookup_leaves_what_lies_between_the_rows_alone():
    base = torch.full((6, 20), 5.0, device="cuda")
    table = torch.ones(4, 9, device="cuda")
    pdb.pdb_embed(pdb.pdb_tokens_create(), table, torch.zeros(6, dtype=torch.int32, device="cuda"), base[:, 3:12])
    assert torch.equal(base[:, :3], torch.full((6, 3), 5.0, device="cuda"))
    assert torch.equal(base[:, 12:], torch.full((6, 8), 5.0, device="cuda"))
    assert torch.equal(base[:, 3:12], torch.ones(6, 9, device="cuda"))


@pytest.mark.parametrize("whole", [torch.int32, torch.int64])
def test_ids_that_are_left_out_and_ids_out_of_range(whole):
    g = _gen(2)
    table = _matrix(10, 16, torch.float32, g)
    table[3] = float("nan")                       # the row of the pad id is not read
    tok = pdb.pdb_tokens_create(8, 16)
    ids = torch.tensor([3, 1, 3, 9], device="cuda", dtype=whole)
    out = torch.full((4, 16), 7.0, device="cuda")
    pdb.pdb_embed(tok, table, ids, out, pad=3)
    assert pdb.pdb_tokens_status(tok) == pdb.PDB_OK
    assert torch.equal(out, torch.where((ids == 3)[:, None], 0.0, table[ids.long().clamp(max=9)]))
    bad = torch.tensor([2, -1, 10, 5], device="cuda", dtype=whole)
    if whole == torch.int64:
        bad[2] = (1 << 32) + 2                    # in range only if cut to 32 bits
    pdb.pdb_embed(tok, table, bad, out, pad=-1)
    assert pdb.pdb_tokens_status(tok) == pdb.PDB_ERANGE
    assert torch.equal(out, torch.stack([table[2], 0 * table[2], 0 * table[2], table[5]]))
    with pytest.raises(pdb.PdbError) as e:
        pdb.check_tokens(tok)
    assert e.value.code == pdb.PDB_ERANGE
    # the error stops no later call, of the gradient's either
    d = torch.ones(4, 16, device="cuda")
    grad = torch.full((10, 16), 9.0, device="cuda")
    pdb.pdb_embed_grad(tok, bad, d, grad, pad=-1)
    want = torch.zeros(10, 16, device="cuda")
    want[2] = want[5] = 1.0
    assert torch.equal(grad, want)
    fresh = pdb.pdb_tokens_create(8, 16)
    pdb.pdb_embed_grad(fresh, ids, d, grad, pad=3)
    assert pdb.pdb_tokens_status(fresh) == pdb.PDB_OK
    want = torch.zeros(10, 16, device="cuda")
    want[1] = want[9] = 1.0
    assert torch.equal(grad, want)
    pdb.pdb_embed_grad(fresh, bad, d, grad, pad=3)
    assert pdb.pdb_tokens_status(fresh) == pdb.PDB_ERANGE


IDS = ["zipf", "uniform", "one", "two", "sorted", "all-left-out"]


def _some_ids(kind, n, vocab, g):
    if kind == "zipf":
        return _zipf(n, vocab, g) if n else torch.zeros(0, dtype=torch.int64, device="cuda")
    if kind == "uniform":
        return torch.randint(0, vocab, (n,), device="cuda", generator=g)
    if kind == "one":
        return torch.full((n,), vocab - 1, device="cuda")
    if kind == "two":
        return torch.randint(0, 2, (n,), device="cuda", generator=g) * (vocab - 1)
    if kind == "sorted":
        return torch.arange(n, device="cuda") * vocab // max(n, 1)
    return torch.full((n,), -1, device="cuda")


def _check_grad(ids, dout, vocab, scale, dtype, accumulate, tok, layout="whole", pad=-1):
    g = _gen(7)
    old = _matrix(vocab, dout.shape[1], dtype, g, layout)
    got = old if layout != "whole" else old.clone()
    keep = old.clone()
    pdb.pdb_embed_grad(tok, ids, dout, got, scale=scale, pad=pad, accumulate=accumulate)
    want, tol = N.embed_grad(ids, dout, vocab, scale, keep if accumulate else None, dtype, pad)
    N.assert_near(got, want, tol, "embed_grad")
    seen = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    inside = ids[(ids != pad) & (ids >= 0) & (ids < vocab)].long()
    seen[inside] = True
    rest = keep[~seen] if accumulate else torch.zeros_like(keep[~seen])
    assert torch.equal(got[~seen], rest)          # rows of ids that do not occur, bit for bit
    return got


@pytest.mark.parametrize("kind", IDS)
@pytest.mark.parametrize("n,vocab,dim", [(0, 5, 8), (1, 1, 1), (31, 40, 3), (32, 1000, 64), (33, 7, 65), (64, 2, 256),
                                         (65, 300, 257), (1000, 10_000, 40), (4096, 50, 24), (4097, 33_000, 8),
                                         (8193, 129, 130)])
def test_gradient(kind, n, vocab, dim):
    g = _gen(3)
    tok = pdb.pdb_tokens_create(n, dim)
    ids = _some_ids(kind, n, vocab, g).to(torch.int32 if n % 2 else torch.int64)
    dout = _matrix(n, dim, torch.float32, g)
    for accumulate in (False, True):
        _check_grad(ids, dout, vocab, -0.37, torch.float32, accumulate, tok)
    pdb.check_tokens(tok)


@pytest.mark.parametrize("a", list(N.TYPES))
@pytest.mark.parametrize("b", list(N.TYPES))
@pytest.mark.parametrize("dim,layout", [(96, "whole"), (96, "shifted"), (101, "padded"), (520, "padded"), (2, "shifted")])
def test_gradient_types_and_layouts(a, b, dim, layout):
    g = _gen(4)
    n, vocab = 700, 90
    tok = pdb.pdb_tokens_create(1000, 600)
    dout = _matrix(n, dim, N.TYPES[a], g, layout)
    ids = _zipf(n, vocab, g)
    for accumulate in (False, True):
        _check_grad(ids, dout, vocab, 1.5, N.TYPES[b], accumulate, tok, layout, pad=int(ids[0]))
    pdb.check_tokens(tok)


@pytest.mark.parametrize("n,vocab,dim,kind", [(70_001, 40_000, 72, "zipf"), (140_000, 3000, 40, "zipf"),
                                              (66_000, 50, 136, "one"), (65_536, 1_000_000, 16, "uniform"),
                                              (200_000, 70_000, 8, "two")])
def test_gradient_of_long_batches(n, vocab, dim, kind):
    g = _gen(5)
    tok = pdb.pdb_tokens_create(n, dim)
    ids = _some_ids(kind, n, vocab, g).int()
    dout = _matrix(n, dim, torch.bfloat16, g)
    first = _check_grad(ids, dout, vocab, 1.0, torch.float32, False, tok)
    again = torch.empty_like(first)
    pdb.pdb_embed_grad(tok, ids, dout, again, scale=1.0)
    assert torch.equal(first, again)              # the same bits every time
    pdb.check_tokens(tok)


def test_gradient_does_not_depend_on_the_other_columns_or_the_handles_size():
    # the order of a run's sums is fixed by the ids alone
    g = _gen(6)
    ids = _zipf(3000, 60, g)
    dout = _matrix(3000, 640, torch.float32, g)
    whole = torch.empty(60, 640, device="cuda")
    pdb.pdb_embed_grad(pdb.pdb_tokens_create(3000, 640), ids, dout, whole)
    for c0, c1 in [(0, 1), (5, 12), (128, 640), (3, 300)]:
        part = torch.empty(60, c1 - c0, device="cuda")
        pdb.pdb_embed_grad(pdb.pdb_tokens_create(10_000, 1000), ids, dout[:, c0:c1], part)
        assert torch.equal(part, whole[:, c0:c1])


def test_gradient_is_the_derivative_of_the_lookup():
    # L = sum(weights * lookup): linear in the table, so a difference of any step is the derivative
    g = _gen(8)
    n, vocab, dim, scale = 50, 12, 6, 3.0
    ids = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    weights = _matrix(n, dim, torch.float32, g)
    table = _matrix(vocab, dim, torch.float32, g)
    tok = pdb.pdb_tokens_create(n, dim)
    grad, out = torch.empty(vocab, dim, device="cuda"), torch.empty(n, dim, device="cuda")
    pdb.pdb_embed_grad(tok, ids, weights, grad, scale=scale)
    for v, j in [(0, 0), (5, 3), (11, 5), (int(ids[0]), 2)]:
        at = []
        for step in (-1.0, 1.0):
            moved = table.clone()
            moved[v, j] += step
            pdb.pdb_embed(tok, moved, ids, out, scale=scale)
            at.append(float((out.double() * weights.double()).sum()))
        # rounding of scale * (table +- 1) to fp32, over the n rows
        tol = 4 * n * 2.0 ** -24 * scale * float(table.abs().max() + 1) * float(weights.abs().max())
        assert abs((at[1] - at[0]) / 2 - float(grad[v, j])) <= tol + 1e-6 * abs(float(grad[v, j]))


def test_ids_at_a_stride():
    g = _gen(31)
    for whole in (torch.int32, torch.int64):
        base = torch.randint(0, 30, (400, 3), device="cuda", generator=g).to(whole)
        ids = base[:, 1]
        table, dout = _matrix(30, 20, torch.float32, g), _matrix(400, 20, torch.float32, g)
        tok = pdb.pdb_tokens_create(400, 20)
        out = torch.empty_like(dout)
        pdb.pdb_embed(tok, table, ids, out)
        assert torch.equal(out, table[ids.long()])
        _check_grad(ids, dout, 30, 1.0, torch.float32, False, tok)
        pdb.check_tokens(tok)


def test_sgd_step_in_place_equals_gradient_then_step():
    g = _gen(9)
    ids, dout = _zipf(500, 100, g), _matrix(500, 48, torch.float32, g)
    tok = pdb.pdb_tokens_create(500, 48)
    table = _matrix(100, 48, torch.float32, g)
    grad = torch.empty_like(table)
    pdb.pdb_embed_grad(tok, ids, dout, grad, scale=-0.25)
    stepped = table + grad
    pdb.pdb_embed_grad(tok, ids, dout, table, scale=-0.25, accumulate=True)
    assert torch.equal(table, stepped)


def test_nan_and_infinity_stay_in_their_rows():
    g = _gen(10)
    ids = torch.randint(0, 20, (300,), device="cuda", generator=g)
    dout = _matrix(300, 40, torch.float32, g)
    dout[7, 3], dout[11, 5] = float("nan"), float("inf")
    grad = torch.empty(20, 40, device="cuda")
    pdb.pdb_embed_grad(pdb.pdb_tokens_create(300, 40), ids, dout, grad)
    odd = ~torch.isfinite(grad)
    want = torch.zeros(20, 40, dtype=torch.bool, device="cuda")
    want[ids[7], 3] = want[ids[11], 5] = True
    assert torch.equal(odd, want)


def test_tables_past_two_to_the_31_elements():
    vocab, dim = 68_000, 32_768                   # 2.2e9 elements of 16 bits
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([67_999, 0, 65_537, 67_999], device="cuda", dtype=torch.int32)
    table[67_999], table[0], table[65_537] = 2.0, 3.0, 4.0
    tok = pdb.pdb_tokens_create(4, dim)
    out = torch.empty(4, dim, dtype=torch.bfloat16, device="cuda")
    pdb.pdb_embed(tok, table, ids, out)
    assert torch.equal(out[:, 0].float().cpu(), torch.tensor([2.0, 3.0, 4.0, 2.0]))
    assert torch.equal(out, out[:, :1].expand_as(out))
    pdb.pdb_embed_grad(tok, ids, out, table, scale=1.0, accumulate=True)
    assert torch.equal(table[[67_999, 0, 65_537, 1]].float().cpu(),
                       torch.tensor([6.0, 6.0, 8.0, 0.0])[:, None].expand(4, dim))
    pdb.check_tokens(tok)


def test_on_another_stream():
    side = torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    table = torch.zeros(100, 512, device="cuda")
    ids = torch.arange(64, device="cuda") % 7
    torch.cuda.synchronize()
    tok = pdb.pdb_tokens_create(64, 512)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-4                # keeps the stream busy before the inputs are written
        table.fill_(2.0)
        out = torch.empty(64, 512, device="cuda")
        pdb.pdb_embed(tok, table, ids, out, scale=3.0)
        grad = torch.empty(100, 512, device="cuda")
        pdb.pdb_embed_grad(tok, ids, out, grad)
    side.synchronize()
    assert torch.equal(out, torch.full_like(out, 6.0))
    count = torch.bincount(ids, minlength=100).float()
    assert torch.equal(grad, (6.0 * count)[:, None].expand_as(grad))
    # the stream given as an argument
    out.zero_()
    torch.cuda.synchronize()
    pdb.pdb_embed(tok, table, ids, out, scale=0.5, stream=side)
    side.synchronize()
    assert torch.equal(out, torch.ones_like(out))


def test_empty_sizes():
    tok = pdb.pdb_tokens_create(4, 8)
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    pdb.pdb_embed(tok, torch.ones(3, 8, device="cuda"), none, torch.empty(0, 8, device="cuda"))
    pdb.pdb_embed(tok, torch.ones(3, 0, device="cuda"), none[:0], torch.empty(0, 0, device="cuda"))
    grad = torch.full((3, 8), 4.0, device="cuda")
    pdb.pdb_embed_grad(tok, none, torch.empty(0, 8, device="cuda"), grad, accumulate=True)
    assert torch.equal(grad, torch.full((3, 8), 4.0, device="cuda"))
    pdb.pdb_embed_grad(tok, none, torch.empty(0, 8, device="cuda"), grad)
    assert torch.equal(grad, torch.zeros(3, 8, device="cuda"))
    pdb.check_tokens(tok)
    # a table without rows: every id is out of range
    pdb.pdb_embed_grad(tok, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.ones(2, 8, device="cuda"),
                       torch.empty(0, 8, device="cuda"))
    assert pdb.pdb_tokens_status(tok) == pdb.PDB_ERANGE


def test_refusals():
    tok = pdb.pdb_tokens_create(10, 16)
    f = lambda *shape, **kw: torch.zeros(*shape, device="cuda", **kw)
    i = lambda n, dtype=torch.int32: torch.zeros(n, device="cuda", dtype=dtype)

    def refused(code, call, *a, **kw):
        with pytest.raises(pdb.PdbError) as e:
            call(*a, **kw)
        assert e.value.code == code, e.value
    both = f(12, 16)
    for a in [(f(4, 16), i(3), f(2, 16)),                      # ids and rows differ
              (f(4, 16), i(3), f(3, 15)),                      # columns differ
              (f(4, 16).double(), i(3), f(3, 16)),             # type
              (f(4, 16), f(3), f(3, 16)),                      # ids of a wrong type
              (f(4, 16), i(3)[:1].expand(3), f(3, 16)),        # ids on top of one another
              (f(4, 16), i(6).view(3, 2), f(6, 16)),           # ids in a matrix
              (f(16, 4).t(), i(3), f(3, 16)),                  # rows not contiguous
              (f(4, 16).cpu(), i(3), f(3, 16)),
              (f(4, 16), i(3).cpu(), f(3, 16)),
              (f(1, 16).expand(4, 16), i(4), f(1, 16).expand(4, 16)),   # rows on top of one another
              (both[:4], i(9), both[3:]),                      # out overlaps the table
              (f(4, 2, 8), i(3), f(3, 16))]:
        refused(pdb.PDB_EINVAL, pdb.pdb_embed, tok, *a)
    for a in [(i(3), f(2, 16), f(4, 16)), (i(3), f(3, 16), f(4, 8)), (i(9), both[3:], both[:4])]:
        refused(pdb.PDB_EINVAL, pdb.pdb_embed_grad, tok, *a)
    refused(pdb.PDB_ETOOBIG, pdb.pdb_embed_grad, tok, i(11), f(11, 16), f(4, 16))
    refused(pdb.PDB_ETOOBIG, pdb.pdb_embed_grad, tok, i(3), f(3, 17), f(4, 17))
    refused(pdb.PDB_EINVAL, pdb.pdb_tokens_create, -1, 4)
    refused(pdb.PDB_ETOOBIG, pdb.pdb_tokens_create, 1 << 31, 4)
    assert pdb.pdb_tokens_status(tok) == pdb.PDB_OK


@pytest.mark.parametrize("n,vocab,dim,layout", [(1, 33, 4100, "whole"), (5, 9045, 880, "whole"), (40, 2100, 4096, "padded"),
                                                (300, 1999, 1200, "shifted"), (2500, 5001, 700, "whole"),
                                                (17_000, 9000, 516, "whole")])
def test_zeroing_by_parts(n, vocab, dim, layout):
    # rows long enough for several warps to share 32 of them, some written beside the sort, and a last group that is not whole
    g = _gen(n)
    tok = pdb.pdb_tokens_create(n, dim)
    ids = _some_ids("zipf", n, vocab, g)
    dout = _matrix(n, dim, torch.float32, g, layout)
    _check_grad(ids, dout, vocab, 0.5, torch.float32, False, tok, layout)
    _check_grad(ids % 32, dout, vocab, 0.5, torch.bfloat16, False, tok, layout)
    pdb.check_tokens(tok)
