"""The gradients of the example's student with experts against differences of its loss, every parameter's.  The loss is the definition's in 64 bits,
at the experts that the student chose: a step of any size changes no choice, and its differences have no noise of their own."""
import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

from tests.test_gpu_tokens_experts import _problem  # noqa: E402

pytestmark = pytest.mark.gpu


def _loss(params, ids, chosen, kept, scale, top_ids, top, lse, T):
    table, out, W, R = params
    n, vocab = ids.shape[0], table.shape[0]
    h = (table[ids] * scale).mean(1)
    p = torch.softmax(h @ R.t(), 1).gather(1, chosen) * kept
    h = h + (torch.einsum("nkij,nj->nki", W[chosen], h) * p[:, :, None]).sum(1)
    logp = torch.log_softmax(h @ out.t() / T, 1)
    q = torch.exp(top.double() / T - lse.double()[:, None])
    inside = torch.zeros(n, vocab, dtype=torch.bool, device="cuda").scatter_(1, top_ids, True)
    rest = 1 - q.sum(1)
    others = torch.logsumexp(logp.masked_fill(inside, -float("inf")), 1)
    return float((T * T * ((q * (q.log() - logp.gather(1, top_ids))).sum(1) + rest * (rest.log() - others))).mean())


def test_gradients_of_all_parameters_by_differences():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.backends.cuda.matmul.allow_tf32 = False
    from examples import token_model as tm
    T = 1.5
    m = tm.Mixed(120, 16, 3, 64, 5, 1.0, experts=4)
    ids, top_ids, top, lse = _problem(vocab=120)
    m.gradients(ids, top_ids, top, lse, T)
    grads = [d.double() for d in m.grads]
    _, _, chosen, place, *_ = m.experts.kept
    params = [w.double() for w in (m.table, m.out, m.experts.W, m.experts.R)]
    compared = 0
    for w, d in zip(params, grads):
        # along the gradient, and along any other direction; what the difference leaves is of the step's third power
        other = torch.randn(w.shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(1))
        for direction in (d, other):
            step = direction / direction.norm() * 1e-4 * w.norm()
            start = w.clone()
            losses = []
            for sign in (1.0, -1.0):
                w.copy_(start + sign * step)
                losses.append(_loss(params, ids, chosen.long(), place >= 0, m.scale, top_ids, top, lse, T))
            w.copy_(start)
            slope, change = float((d * step).sum()), (losses[0] - losses[1]) / 2
            # every element of a gradient is good to 1e-4 of the largest (products of up to 120 terms and sums of up to 60 rows in fp32)
            off = 1e-4 * float(d.abs().max() * step.abs().sum())
            assert abs(change - slope) <= off + 1e-6 * abs(slope)
            if direction is d:
                assert abs(slope) > 10 * off
                compared += 1
    assert compared == 4
