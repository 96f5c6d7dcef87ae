"""The operators together as the example uses them: a student with experts whose clipped step is held against automatic differentiation in 64
bits, its training, a recorded step, and its drafts for the teacher."""
import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()
    torch.backends.cuda.matmul.allow_tf32 = False


def _problem(n=64, vocab=300, context=3, seed=6):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, vocab, (n, context), device="cuda", generator=g)
    ids[:20] = 7
    teacher = torch.randn(n, vocab, device="cuda", generator=g) * 2
    top, top_ids = torch.topk(teacher, 10, dim=1)
    return ids, top_ids, top, torch.logsumexp(teacher / 1.5, 1)


@pytest.mark.parametrize("max_norm", [0.05, 1e6])
def test_a_step_is_clipped_sgd_on_the_loss(max_norm):
    from examples import token_model as tm
    m = tm.Mixed(300, 16, 3, 64, 5, 1.0, experts=6, max_norm=max_norm)
    ids, top_ids, top, lse = _problem()
    T, eta = 1.5, 0.5
    table, out, W, R = params = [w.double().requires_grad_() for w in (m.table, m.out, m.experts.W, m.experts.R)]
    loss = m.gradients(ids, top_ids, top, lse, T)
    grads = [d.clone() for d in m.grads]
    # the experts that the step chose, without the slots behind an expert's capacity
    _, _, chosen, place, *_ = m.experts.kept
    h = (table[ids] * m.scale).mean(1)
    p = torch.softmax(h @ R.t(), 1).gather(1, chosen.long()) * (place >= 0)
    assert (place < 0).sum() < place.numel() // 4
    h2 = h + (torch.einsum("nkij,nj->nki", W[chosen.long()], h) * p[:, :, None]).sum(1)
    logp = torch.log_softmax(h2 @ out.t() / T, 1)
    q = torch.exp(top.double() / T - lse.double()[:, None])
    inside = torch.zeros(64, 300, dtype=torch.bool, device="cuda").scatter_(1, top_ids, True)
    rest = 1 - q.sum(1)
    kl = (q * (q.log() - logp.gather(1, top_ids))).sum(1) + rest * (rest.log() - torch.logsumexp(logp.masked_fill(inside, -float("inf")), 1))
    want = T * T * kl
    exact = torch.autograd.grad(want.mean(), params)
    # products of up to 300 terms and sums of up to 60 rows in fp32, one after the other: 1e-4 of the largest gradient covers them
    assert torch.allclose(loss.double(), want, rtol=1e-4, atol=1e-5)
    for got, d in zip(grads, exact):
        assert (got.double() - d).abs().max() <= 1e-4 * d.abs().max()
    m.step(ids, top_ids, top, lse, T, eta)
    norm = torch.sqrt(sum((d ** 2).sum() for d in exact))
    assert abs(float(m.norm) - float(norm)) <= 1e-4 * float(norm)
    f = min(1.0, max_norm / float(norm))
    assert (f < 1.0) == (max_norm < 1.0)
    for w, start, d in zip((m.table, m.out, m.experts.W, m.experts.R), params, exact):
        assert (w.double() - start.detach() + eta * f * d).abs().max() <= 1e-4 * eta * f * d.abs().max() + 2e-7
    pdb.check_tokens(m.tok)
    pdb.check_tokens(m.experts.tok)


def test_gradients_by_differences():
    from examples import token_model as tm
    m = tm.Mixed(120, 16, 3, 64, 5, 1.0, experts=4)
    ids, top_ids, top, lse = _problem(vocab=120)
    m.gradients(ids, top_ids, top, lse, 1.5)
    grads = [d.clone() for d in m.grads]
    place = m.experts.kept[3].clone()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for w, d in zip((m.table, m.out, m.experts.W, m.experts.R), grads):
        # along the gradient itself, where the change is largest; second differences cancel, and the loss is good to about 1e-6
        step = d / d.norm() * 1e-2 * w.norm() / w.numel() ** 0.5
        losses = []
        for sign in (1.0, -1.0):
            w += sign * step
            losses.append(float(m.gradients(ids, top_ids, top, lse, 1.5).double().mean()))
            same = torch.equal(m.experts.kept[3], place)
            w -= sign * step
            if not same:
                break
        if same:                                       # no example changed its experts
            slope = float((d.double() * step.double()).sum())
            assert abs((losses[0] - losses[1]) / 2 - slope) <= 0.02 * abs(slope) + 2e-6


def test_training_runs():
    from examples import token_model as tm
    models = []
    losses, before, after, best = tm.train(steps=20, vocab=300, dim=32, tokens=256, experts=8, models=models)
    assert len(losses) >= 2 and all(x == x for x in losses)
    text, accepted = tm.speculate(models[0], models[1], torch.randint(0, 300, (32, 4), device="cuda"), rounds=3)
    assert text.shape == (32, 3, 5) and accepted.shape == (32, 3)
    there = (text >= 0).sum(2)
    assert torch.equal(there, accepted.long() + 1) and int(text.max()) < 300


def test_a_step_in_a_graph():
    from examples import token_model as tm
    a, b = (tm.Mixed(300, 16, 3, 64, 5, 1.0, experts=6, max_norm=0.1) for _ in range(2))
    ids, top_ids, top, lse = _problem()
    for _ in range(2):                                 # the first calls choose the products' algorithms
        a.step(ids, top_ids, top, lse, 1.5, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(ids, top_ids, top, lse, 1.5, 0.5)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(ids, top_ids, top, lse, 1.5, 0.5)
    graph.replay()
    for x, y in zip((a.table, a.out, a.experts.W, a.experts.R), (b.table, b.out, b.experts.W, b.experts.R)):
        assert (x - y).abs().max() <= 1e-5 * x.abs().max()


def test_drafts_leave_the_targets_distribution():
    # first and second tokens of many sequences against the target's probabilities: counts lie within 5 standard deviations
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    n, V, D = 200_000, 12, 2
    z = torch.randn(D + 1, V, device="cuda", generator=g) * 1.5
    y = torch.randn(D, V, device="cuda", generator=g) * 1.5
    tok = pdb.pdb_tokens_create(0, 0)
    draft = y.repeat(n, 1)
    drawn = torch.empty(n * D, 1, device="cuda", dtype=torch.int32)
    none = torch.empty(n * D, 0, device="cuda")
    pdb.pdb_verify(tok, draft, none.int(), none, torch.rand(n * D, device="cuda", generator=g), drawn)
    tokens, accepted = torch.empty(n, D + 1, device="cuda", dtype=torch.int32), torch.empty(n, device="cuda", dtype=torch.int32)
    pdb.pdb_verify(tok, z.repeat(n, 1), drawn.view(n, D), torch.rand(n, D, device="cuda", generator=g),
                   torch.rand(n, device="cuda", generator=g), tokens, accepted, draft=draft)
    q = torch.softmax(y.double(), 1)
    for d in range(D + 1):
        at = tokens[:, d][tokens[:, d] >= 0].long()
        p = torch.softmax(z[d].double(), 0)
        share = torch.bincount(at, minlength=V).double() / at.numel()
        assert ((share - p).abs() <= 5 * torch.sqrt(p * (1 - p) / at.numel())).all()
        if d < D:
            taken = torch.minimum(p, q[d]).sum()          # of the sequences that reach the position
            reach = int((accepted >= d).sum())
            got = int((accepted > d).sum()) / reach
            assert abs(got - float(taken)) <= 5 * float(torch.sqrt(taken * (1 - taken) / reach))
