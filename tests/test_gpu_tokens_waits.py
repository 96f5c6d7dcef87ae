"""Waits of pdb_distill's gradient that run out: without a try the readers give up at once, so the warp that brings the
rows finds no place free after the first ones.  The call ends and says so, and calls after it are as ever."""
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


def _problem(n, cols, K, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn(n, cols, device="cuda", generator=g).to(dtype)
    top, ids = torch.topk(z.float() + torch.randn(n, cols, device="cuda", generator=g), K, dim=1)
    return z, ids, top, torch.logsumexp(torch.cat([top, top[:, :1] + 1], 1), 1)


# blocks of 64, 128 and 256 threads, alone and in clusters of two, four and eight; many rows a cluster and fewer rows than
# clusters; rows that fit in their places and rows that pass through them
@pytest.mark.parametrize("n,cols,K,kind", [
    (1500, 3001, 9, "bf16"), (900, 20_001, 33, "f16"), (700, 40_000, 200, "bf16"), (700, 130_001, 5, "bf16"),
    (400, 100_000, 64, "f32"), (3, 600_000, 50, "bf16"), (2, 1 << 21, 1024, "f32"), (1, 7, 3, "f32")])
@pytest.mark.parametrize("bucket", [False, True])
def test_expired_waits_are_reported_not_hung(n, cols, K, kind, bucket):
    z, ids, top, lse = _problem(n, cols, K, N.TYPES[kind], cols)
    lse = lse if bucket else None
    guard = torch.full((n, cols + 16), 7.0, device="cuda", dtype=z.dtype)
    d, loss = guard[:, 8:8 + cols], torch.empty(n, device="cuda")
    tok = pdb.pdb_tokens_create()
    pdb.pdb_tokens_set_wait_limit(tok, 0)
    for _ in range(2):
        pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, dlogits=d)
    assert pdb.pdb_tokens_status(tok) == pdb.PDB_ETIMEOUT
    assert (guard[:, :8] == 7.0).all() and (guard[:, 8 + cols:] == 7.0).all()
    own = z.clone()
    pdb.pdb_distill(tok, own, ids, top, loss, teacher_lse=lse, dlogits=own)
    with pytest.raises(pdb.PdbError) as e:
        pdb.check_tokens(tok)
    assert e.value.code == pdb.PDB_ETIMEOUT
    # the device works on, with the same handle once it may wait again
    pdb.pdb_tokens_set_wait_limit(tok, 1 << 22)
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, dlogits=d)
    rows = slice(max(0, n - 4), n)
    (want, tol), (grad, tol_g) = N.distill(z[rows], ids[rows], top[rows], None if lse is None else lse[rows], 1.0, None,
                                           z.dtype)
    N.assert_near(loss[rows], want, tol, "loss")
    N.assert_near(d[rows], grad, tol_g, "dlogits")


def test_limits_refused():
    tok = pdb.pdb_tokens_create()
    for tries in (-1, (1 << 22) + 1, 1 << 31):
        with pytest.raises(pdb.PdbError) as e:
            pdb.pdb_tokens_set_wait_limit(tok, tries)
        assert e.value.code == pdb.PDB_EINVAL


def test_calls_that_do_not_wait_take_no_notice():
    tok = pdb.pdb_tokens_create(64, 8)
    pdb.pdb_tokens_set_wait_limit(tok, 0)
    z, ids, top, _ = _problem(5, 300, 4, torch.float32, 1)
    loss = torch.empty(5, device="cuda")
    pdb.pdb_distill(tok, z, ids, top, loss)
    pdb.pdb_logprobs(tok, z, lse=loss)
    grad = torch.empty(10, 8, device="cuda")
    pdb.pdb_embed_grad(tok, torch.zeros(64, dtype=torch.int32, device="cuda"), torch.ones(64, 8, device="cuda"), grad)
    assert grad[0].tolist() == [64.0] * 8
    pdb.check_tokens(tok)
