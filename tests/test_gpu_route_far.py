"""Tokens to experts and back with one slot a token, rows of several widths, and matrices of more than 2^31 elements: without weights what comes back is
what went there, and the rows' gradient is the tokens' at their places."""
import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

from tests.test_gpu_route import _gen, tok, test_join, test_join_grad, test_rows  # noqa: E402,F401

pytestmark = pytest.mark.gpu
there, back, gradients = test_rows, test_join, test_join_grad
del test_rows, test_join, test_join_grad


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.mark.parametrize("n,experts,capacity,dim", [(700, 8, 0, 64), (700, 8, 100, 1001), (1000, 64, 0, 250), (33, 4, 9, 4104), (257, 16, 0, 2048)])
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16")])
def test_one_slot(tok, n, experts, capacity, dim, a, b):  # noqa: F811
    there(tok, n, 1, experts, capacity, dim, a, b)
    back(tok, n, 1, experts, capacity, dim, a, b, True)
    for form in ("all", "in place", "rows alone"):
        gradients(tok, n, 1, experts, capacity, dim, a, b, form)


@pytest.mark.parametrize("dim", [4104, 4101])
def test_more_than_2_31_elements(dim):
    n, experts = 530_000, 64
    g = _gen(dim)
    x = torch.randn(n, dim, device="cuda", generator=g, dtype=torch.bfloat16)
    assert x.numel() > 1 << 31
    ids = torch.randint(0, experts, (n, 1), device="cuda", generator=g, dtype=torch.int32)
    mine = pdb.pdb_tokens_create(n, 0)
    place, source = torch.empty(n, 1, device="cuda", dtype=torch.int32), torch.empty(n, device="cuda", dtype=torch.int32)
    ends = torch.empty(experts, device="cuda", dtype=torch.int32)
    pdb.pdb_route(mine, ids, experts, place, source, ends)
    assert torch.equal(source.long(), torch.sort(ids[:, 0], stable=True).indices)
    rows, y = torch.empty_like(x), torch.empty_like(x)
    pdb.pdb_route_rows(mine, x, place, source, rows)
    assert torch.equal(rows, x[source.long()])
    pdb.pdb_route_join(mine, rows, place, y)
    assert torch.equal(y, x)
    dweight = torch.empty(n, 1, device="cuda")
    y.zero_()
    pdb.pdb_route_join_grad(mine, rows, place, source, x, y, dweight=dweight)
    assert torch.equal(y, rows)
    some = torch.tensor([0, 1, n // 2, n - 1], device="cuda")
    # dim products of like numbers in fp32: dim u of their sum at most
    want = x[some].double().square().sum(1)
    assert ((dweight[some, 0].double() - want).abs() <= dim * 2.0 ** -24 * want).all()
    pdb.check_tokens(mine)
