"""pdb_verify of hundreds of sequences with long rows: clusters of four blocks, of two and of one, by the number of sequences, and of as many as their
pieces need; against the definition in 64 bits, as in test_gpu_verify.py."""
import pytest

from tests._tokens import TYPES

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

from tests.test_gpu_verify import _call, _check, _gen, _inputs, _softmax, _want  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create(0, 0)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,vocab", [(200, 20_011), (400, 10_007), (700, 12_345)])
@pytest.mark.parametrize("lookup", [False, True])
def test_hundreds_of_sequences(tok, kind, n, vocab, lookup):
    _check(tok, *_inputs(n, 1, vocab, TYPES[kind], seed=n, lookup=lookup, ragged=True))
    pdb.check_tokens(tok)


def _repeated(tok, few, n, kind, vocab, D, seed):
    """n sequences in which the `few` first ones come again and again, each time with numbers of their own."""
    z, ids, _, _, y = _inputs(few, D, vocab, TYPES[kind], seed=seed)
    again = torch.arange(n, device="cuda") % few
    g = _gen(seed + 1)
    u, v = torch.rand(n, D, device="cuda", generator=g), torch.rand(n, device="cuda", generator=g)
    z = z.view(few, D + 1, vocab)[again].view(n * (D + 1), vocab)
    y = y.view(few, D, vocab)[again].view(n * D, vocab) if D else None
    return z, ids[again], u, v, y


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("vocab", [600_001, (1 << 21) - 3, 1 << 21])
def test_long_rows_of_many_sequences(tok, kind, vocab):
    # one more than what gives a cluster one block: its pieces have no room in one block's shared memory from 1.8 million tokens on
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n = 4 * sms + 1
    z, ids, u, v, _ = _repeated(tok, 2, n, kind, vocab, 0, 5)
    tokens, accepted, _ = _call(tok, z, ids, u, v, None)
    for row in range(2):
        p = _softmax(z[row], 1.0)
        upto = p.cumsum(0)
        assert torch.equal(tokens[row::2, 0].cpu().long(), torch.searchsorted(upto, v[row::2].double().cpu() * upto[-1], right=True))
    assert (accepted == 0).all()


@pytest.mark.parametrize("n", [160, 310])
def test_long_rows_with_drafts(tok, n):
    # 1.2 million tokens: two blocks have no room for three of their kind on an SM
    args = _repeated(tok, 4, n, "bf16", 1_200_000, 1, 6)
    tokens, accepted, _ = _call(tok, *args)
    z, ids, u, v, y = args
    some = torch.arange(0, n, 9, device="cuda")
    want, count = _want(z.view(n, 2, -1)[some].view(2 * some.numel(), -1), ids[some], u[some], v[some], y[some])
    assert torch.equal(tokens[some].cpu(), want) and torch.equal(accepted[some].cpu(), count)
