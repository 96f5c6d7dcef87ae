"""The token operators together: the example's training step against automatic
differentiation in 64 bits, its training, the operators inside a CUDA graph, and
vocabularies and batches at the ends of their ranges."""
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


def test_a_training_step_is_sgd_on_the_loss():
    from examples import token_model as tm
    torch.backends.cuda.matmul.allow_tf32 = False
    m = tm.Model(300, 16, 3, 64, 5, 1.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    ids = torch.randint(0, 300, (64, 3), device="cuda", generator=g)
    ids[:20] = 7                                   # an id that most of the batch shares
    teacher = torch.randn(64, 300, device="cuda", generator=g) * 2
    top, top_ids = torch.topk(teacher, 10, dim=1)
    T, eta = 1.5, 0.5
    lse = torch.logsumexp(teacher / T, 1)
    table, out = m.table.double().requires_grad_(), m.out.double().requires_grad_()
    h = (table[ids] * m.scale).mean(1)
    logp = torch.log_softmax(h @ out.t() / T, 1)
    q = torch.exp(top.double() / T - lse.double()[:, None])
    inside = torch.zeros(64, 300, dtype=torch.bool, device="cuda").scatter_(1, top_ids, True)
    rest = 1 - q.sum(1)
    kl = (q * (q.log() - logp.gather(1, top_ids))).sum(1)
    kl = kl + rest * (rest.log() - torch.logsumexp(logp.masked_fill(inside, -math.inf), 1))
    want = T * T * kl
    dtable, dout = torch.autograd.grad(want.mean(), (table, out))
    loss = m.step(ids, top_ids, top, lse, T, eta)
    # products of 300 and 64 terms and sums of up to 60 rows in fp32: 1e-4 of the largest change covers them
    assert torch.allclose(loss.double(), want, rtol=1e-4, atol=1e-5)
    for got, start, grad in ((m.table, table, dtable), (m.out, out, dout)):
        change = got.double() - start.detach()
        assert (change + eta * grad).abs().max() <= 1e-4 * eta * grad.abs().max() + 2e-7
    pdb.check_tokens(m.tok)


def test_the_example_learns():
    from examples import token_model as tm
    losses, before, after, best = tm.train(steps=400, vocab=500, dim=32, tokens=512)
    assert losses[-1] < 0.5 * losses[0]
    assert after[0] > before[0] + 0.5 * (best[0] - before[0])      # more than half of the way to the teacher
    assert after[2] > before[2]


def test_inside_a_cuda_graph():
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    n, vocab, dim = 3000, 4000, 48                  # ids of the sort by a cluster
    tok = pdb.pdb_tokens_create(n, dim)
    ids = torch.randint(0, vocab, (n,), device="cuda", generator=g)
    table = torch.randn(vocab, dim, device="cuda", generator=g)
    rows, grad = torch.empty(n, dim, device="cuda"), torch.empty(vocab, dim, device="cuda")
    z = torch.randn(40, vocab, device="cuda", generator=g)
    top, top_ids = torch.topk(z + torch.randn(40, vocab, device="cuda", generator=g), 8, dim=1)
    out = dict(logp=torch.empty(40, device="cuda"), lse=torch.empty(40, device="cuda"),
               entropy=torch.empty(40, device="cuda"), top_ids=torch.empty(40, 6, device="cuda", dtype=torch.int32))
    loss, d1, d2 = torch.empty(40, device="cuda"), torch.empty_like(z), torch.empty_like(z)

    def run():
        pdb.pdb_embed(tok, table, ids, rows)
        pdb.pdb_embed_grad(tok, ids, rows, grad)
        pdb.pdb_logprobs(tok, z, ids[:40], **out)
        pdb.pdb_logprobs_grad(tok, z, ids[:40], out["lse"], None, loss, None, d1)
        pdb.pdb_distill(tok, z, top_ids, top, loss, dlogits=d2)
    loss.fill_(0.5)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    loss.fill_(0.5)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run()
    for _ in range(2):
        # other contents of the same tensors
        ids.copy_(torch.randint(0, vocab, (n,), device="cuda", generator=g))
        z.copy_(torch.randn(40, vocab, device="cuda", generator=g))
        loss.fill_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (rows, grad, *out.values(), loss, d1, d2)]
        for t in (rows, grad, d1, d2):
            t.zero_()
        loss.fill_(0.5)
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (rows, grad, *out.values(), loss, d1, d2)))
        want, tol = N.embed_grad(ids, rows, vocab, 1.0)
        N.assert_near(grad, want, tol, "embed_grad")
    pdb.check_tokens(tok)


@pytest.mark.parametrize("kind,cols", [("f32", 1 << 21), ("bf16", 1_500_001), ("f32", 450_000)])
def test_the_longest_rows(kind, cols):
    # shares of a row that no block can hold, and the most marks that a block has room for
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    tok = pdb.pdb_tokens_create()
    z = torch.randn(2, cols, device="cuda", generator=g).to(N.TYPES[kind])
    top, ids = torch.topk(z.float() + torch.randn(2, cols, device="cuda", generator=g), 1024, dim=1)
    lse = torch.logsumexp(torch.cat([top, top[:, :1] + 8], 1), 1)
    (want, tol), (grad, tol_g) = N.distill(z, ids, top, lse, 1.0, None, z.dtype)
    loss, d = torch.empty(2, device="cuda"), torch.empty_like(z)
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse)
    N.assert_near(loss, want, tol, "loss")
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, dlogits=d)
    N.assert_near(loss, want, tol, "loss beside the gradient")
    N.assert_near(d, grad, tol_g, "dlogits")
    with pytest.raises(pdb.PdbError) as e:
        wide = torch.zeros(1, (1 << 21) + 1, device="cuda")
        pdb.pdb_distill(tok, wide, ids[:1], top[:1], loss[:1])
    assert e.value.code == pdb.PDB_ETOOBIG
    pdb.check_tokens(tok)


@pytest.mark.parametrize("n", [1025, 2048, 2049, 8192, 8193, 16_385, 32_769, 65_536, 65_537])
@pytest.mark.parametrize("vocab", [3, 1000, 70_000, 3_000_000])
def test_sorts_at_their_limits(n, vocab):
    # one column: the sums show each id's rows, and the order of the rows within it by the weights
    g = torch.Generator(device="cuda")
    g.manual_seed(n + vocab)
    tok = pdb.pdb_tokens_create(n, 1)
    ids = torch.randint(-1, vocab, (n,), device="cuda", generator=g)
    d = torch.randint(-8, 9, (n, 1), device="cuda", generator=g).float()      # sums exact in fp32
    grad = torch.empty(vocab, 1, device="cuda")
    pdb.pdb_embed_grad(tok, ids, d, grad)
    want = torch.zeros(vocab + 1, device="cuda").index_add_(0, ids % (vocab + 1), d[:, 0])[:vocab]
    assert torch.equal(grad[:, 0], want)
    pdb.check_tokens(tok)


def test_rows_of_many_clusters():
    # more rows than clusters at once, rows of odd length, both visits of the stream, marks set and cleared row after row
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    for n, cols, K in ((1500, 3001, 9), (700, 130_001, 5)):
        tok = pdb.pdb_tokens_create()
        z = torch.randn(n, cols, device="cuda", generator=g).bfloat16()
        top, ids = torch.topk(z.float() + torch.randn(n, cols, device="cuda", generator=g), K, dim=1)
        lse = torch.logsumexp(torch.cat([top, top[:, :1] - 1], 1), 1)
        loss, d = torch.empty(n, device="cuda"), torch.empty_like(z)
        pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, dlogits=d)
        for rows in (slice(0, 8), slice(n // 2, n // 2 + 8), slice(n - 8, n)):
            (want, tol), (grad, tol_g) = N.distill(z[rows], ids[rows], top[rows], lse[rows], 1.0, None, z.dtype)
            N.assert_near(loss[rows], want, tol, "loss")
            N.assert_near(d[rows], grad, tol_g, "dlogits")
        # every row, by the gradient's own sum: the parts outside and inside of the slots cancel
        total = d.float().sum(1).abs()
        assert float(total.max()) < 2e-2
        pdb.check_tokens(tok)
