"""pdb_distill where the student masks tokens by its type's lowest value: a teacher's token among them costs a loss of 1e37 and
more, finite where T^2 q z is, and the gradient is finite whatever is masked."""
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


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("bucket", [False, True])
@pytest.mark.parametrize("temperature", [0.05, 0.3, 0.6, 0.99, 1.0])
@pytest.mark.parametrize("cols", [70, 2003, 150_001])
def test_masked_slots(kind, bucket, temperature, cols):
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    n, K = 6, 8
    dtype = N.TYPES[kind]
    low = torch.finfo(dtype).min
    z = torch.randn(n, cols, device="cuda", generator=g).to(dtype)
    top, ids = torch.topk(z.float() + torch.randn(n, cols, device="cuda", generator=g) * 0.3, K, dim=1)
    lse = torch.logsumexp(torch.cat([top, top[:, :1]], 1) / temperature, 1) if bucket else None
    z[1, ids[1, 3]] = low                              # one slot
    z[2, ids[2]] = low                                 # every slot
    z[3, torch.rand(cols, device="cuda", generator=g) < 0.5] = low
    z[4] = low                                         # everything: uniform
    outside = torch.ones(cols, dtype=torch.bool, device="cuda")
    outside[ids[5]] = False
    z[5, outside] = low                                # all but the slots
    tok = pdb.pdb_tokens_create()
    (want, tol), (grad, tol_g) = N.distill(z, ids, top, lse, temperature, None, dtype)
    loss, d = torch.empty(n, device="cuda"), torch.empty_like(z)
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, temperature=temperature)
    N.assert_near(loss, want, tol, "loss")
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, temperature=temperature, dlogits=d)
    N.assert_near(loss, want, tol, "loss beside the gradient")
    assert torch.isfinite(d).all()
    rows = [0, 1, 2, 3, 4]
    N.assert_near(d[rows], grad[rows], tol_g[rows], "dlogits")
    # row 5: outside of the slots p is 0 and p / p_t is 1 / (cols - K)
    T = float(torch.tensor(temperature, dtype=torch.float32))
    rest = float(1 - torch.exp(top[5].double() / T - lse[5].double()).sum()) if bucket else 0.0
    flat = torch.full((cols - K,), -T * rest / (cols - K), dtype=torch.float64)
    bound = N.SLACK * N.U * T * (3 * float(top[5].abs().max()) / T + 64 + N.terms(cols)) / (cols - K)
    N.assert_near(d[5, outside], flat, bound + N.rounding(flat, dtype), "outside of the slots")


@pytest.mark.parametrize("bucket", [False, True])
def test_infinite_and_empty_below_a_temperature_of_one(bucket):
    # what is infinite stays so, and a row without slots to learn from has loss 0, also where the slots hold every token
    z = torch.randn(4, 6, device="cuda")
    z[0, 2] = -float("inf")                            # a slot that the student rules out
    z[1] = -float("inf")
    ids = torch.arange(6, device="cuda").repeat(4, 1)
    top = torch.zeros(4, 6, device="cuda")
    top[2] = -float("inf")
    ids[3] = -1
    lse = torch.full((4,), 9.0, device="cuda") if bucket else None
    loss, d = torch.empty(4, device="cuda"), torch.empty_like(z)
    tok = pdb.pdb_tokens_create()
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, temperature=0.5, dlogits=d)
    assert loss.tolist() == [float("inf")] * 2 + [0.0] * 2
    assert torch.count_nonzero(d[1:]) == 0
    alone = torch.empty(4, device="cuda")
    pdb.pdb_distill(tok, z, ids, top, alone, teacher_lse=lse, temperature=0.5)
    assert torch.equal(alone, loss)
