"""Matrices whose rows lie between one another's rows, as column ranges of one buffer do, share no memory: every call takes
them and gives the bits that it gives for matrices apart, and writes nothing else."""
import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create(4096, 512)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _in_turn(rows, cols, dtype, gap, first):
    """A buffer of `rows` rows with two ranges of `cols` columns, `gap` apart, from column `first` on."""
    whole = torch.full((rows, first + 2 * cols + gap + 3), 7.0, device="cuda", dtype=dtype)
    a, b = whole[:, first:first + cols], whole[:, first + cols + gap:first + 2 * cols + gap]
    rest = torch.ones(whole.shape[1], dtype=torch.bool, device="cuda")
    rest[first:first + cols] = False
    rest[first + cols + gap:first + 2 * cols + gap] = False
    return whole, a, b, rest


LAYOUTS = [(0, 0), (0, 8), (5, 0), (3, 1)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("gap,first", LAYOUTS)
@pytest.mark.parametrize("n,cols", [(2, 5), (37, 1000), (9, 20_001)])
def test_gradients_beside_their_logits(tok, kind, gap, first, n, cols):
    g = _gen(cols)
    z = torch.randn(n, cols, device="cuda", generator=g).to(TYPES[kind])
    ids = torch.randint(0, cols, (n,), device="cuda", generator=g)
    top, slots = torch.topk(z.float() + torch.randn(n, cols, device="cuda", generator=g), 4, dim=1)
    lse, H = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    pdb.pdb_logprobs(tok, z, lse=lse, entropy=H)
    a, b, loss = (torch.randn(n, device="cuda", generator=g) for _ in range(3))
    apart = _in_turn(n, cols, z.dtype, gap, first)[2]       # of the same alignment, in a buffer of its own
    for call in (lambda z, d: pdb.pdb_logprobs_grad(tok, z, ids, lse, H, a, b, d),
                 lambda z, d: pdb.pdb_distill(tok, z, slots, top, loss, dlogits=d)):
        whole, logits, d, rest = _in_turn(n, cols, z.dtype, gap, first)
        logits.copy_(z)
        call(logits, d)
        call(_in_turn(n, cols, z.dtype, gap, first)[1].copy_(z), apart)
        assert torch.equal(d, apart) and torch.equal(logits, z) and (whole[:, rest] == 7.0).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("gap,first", LAYOUTS)
def test_rows_beside_their_table(tok, kind, gap, first):
    g = _gen(3)
    vocab, dim, n = 300, 96, 200
    whole, table, out, rest = _in_turn(vocab, dim, TYPES[kind], gap, first)
    table.copy_(torch.randn(vocab, dim, device="cuda", generator=g))
    given = table.clone()
    ids = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    pdb.pdb_embed(tok, table, ids, out[:n], scale=2.0)
    assert torch.equal(out[:n], (given[ids].float() * 2.0).to(given.dtype))
    assert torch.equal(table, given) and (out[n:] == 7.0).all() and (whole[:, rest] == 7.0).all()
    rows = out[:n].clone()
    for accumulate in (False, True):
        want = given.clone()
        pdb.pdb_embed_grad(tok, ids, rows, want, accumulate=accumulate)
        table.copy_(given)
        pdb.pdb_embed_grad(tok, ids, out[:n], table, accumulate=accumulate)
        assert torch.equal(table, want) and torch.equal(out[:n], rows)
        assert (out[n:] == 7.0).all() and (whole[:, rest] == 7.0).all()


def test_rows_of_other_strides(tok):
    # every second row of a table is the result's
    buffer = torch.arange(64 * 8, device="cuda", dtype=torch.float32).view(64, 8)
    given = buffer.clone()
    table, out = buffer[::4], buffer[1::2]                  # strides 32 and 16: rows 0, 4, 8, ... and 1, 3, 5, ...
    ids = torch.arange(16, device="cuda").repeat(2)
    pdb.pdb_embed(tok, table, ids, out)
    assert torch.equal(out, given[::4][ids]) and torch.equal(buffer[::2], given[::2])
    with pytest.raises(pdb.PdbError) as e:
        pdb.pdb_embed(tok, table, ids[:16], buffer[::2][:16])
    assert e.value.code == pdb.PDB_EINVAL
    pdb.check_tokens(tok)
