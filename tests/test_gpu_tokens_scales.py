"""Scales and temperatures up to where they are refused: finite results, by the definition in 64 bits."""
import math

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


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e10, 1e30, 2.3e38])
def test_log_probabilities(scale):
    # two equal tokens above the others: at a large scale half each, at a small one all alike
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tok = pdb.pdb_tokens_create()
    z = -torch.rand(3, 1000, device="cuda", generator=g) - 0.5
    z[:, 10], z[:, 700] = 0.0, 0.0
    z[1] += 3.0
    ids = torch.full((3,), 10, device="cuda")
    out = {m: torch.empty(3, device="cuda") for m in ("logp", "lse", "entropy")}
    pdb.pdb_logprobs(tok, z, ids, scale=scale, **out)
    n = 2 if scale > 1 else 1000
    bound = 2 * N.U * (N.terms(1000) + 8) * (math.log(n) + 1)
    assert (out["logp"].double() + math.log(n)).abs().max() <= bound
    assert (out["entropy"].double() - math.log(n)).abs().max() <= bound
    a, d = torch.ones(3, device="cuda"), torch.empty_like(z)
    pdb.pdb_logprobs_grad(tok, z, ids, out["lse"], None, a, None, d, scale=scale)
    s = float(torch.tensor(scale, dtype=torch.float32))
    want = torch.zeros(3, 1000, dtype=torch.float64)
    want[:, [10, 700] if scale > 1 else slice(None)] = -s / n
    want[:, 10] += s
    N.assert_near(d, want, s * 2 * N.U * (N.terms(1000) + 64) * torch.ones_like(want), "dlogits")


@pytest.mark.parametrize("temperature", [1e-12, 1e-3, 1e3])
@pytest.mark.parametrize("bucket", [False, True])
def test_distillation(temperature, bucket):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    tok = pdb.pdb_tokens_create()
    z = torch.randn(4, 900, device="cuda", generator=g) * temperature          # of the temperature's size
    top, ids = torch.topk(z + torch.randn(4, 900, device="cuda", generator=g) * temperature, 6, dim=1)
    T = float(torch.tensor(temperature, dtype=torch.float32))
    lse = torch.logsumexp(torch.cat([top, top[:, :1]], 1) / T, 1) if bucket else None
    (want, tol), (grad, tol_g) = N.distill(z, ids, top, lse, temperature)
    loss, d = torch.empty(4, device="cuda"), torch.empty_like(z)
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, dlogits=d, temperature=temperature)
    N.assert_near(loss, want, tol, "loss")
    N.assert_near(d, grad, tol_g, "dlogits")
