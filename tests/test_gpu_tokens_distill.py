"""pdb_distill's loss and gradient against the definition in 64 bits, with bounds
from fp32 rounding (tests/_tokens.py), and the gradient against differences:
slots that are empty, repeated or masked, with and without the bucket for the
teacher's rest, a student surer than fp32 can tell by subtraction, every type."""
import math

import pytest

from tests import _tokens as N

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lay(z, layout):
    if layout == "whole":
        return z
    base = torch.full((z.shape[0], z.shape[1] + 5), 1e4, device="cuda").to(z.dtype)
    base[:, 3:3 + z.shape[1]] = z
    return base[:, 3:3 + z.shape[1]]


def _problem(n, cols, K, dtype, g, temperature=1.0, top_type=torch.float32, wide=True):
    z = (torch.randn(n, cols, device="cuda", generator=g) * 2).to(dtype)
    teacher = z.float() + torch.randn(n, cols, device="cuda", generator=g)
    top, ids = torch.topk(teacher, K, dim=1)
    # what a slot loses in rounding to its type must not lift the slots above the whole: a little more in the rest
    lse = torch.logsumexp(torch.cat([teacher, top[:, :1] - 1.0], 1) / temperature, 1)
    return z, (ids if wide else ids.int()), top.to(top_type), lse


def _check(tok, z, ids, top, lse, temperature=1.0, weight=None, layout="whole", inplace=False, with_loss=True):
    n = z.shape[0]
    (want, tol), (grad, tol_g) = N.distill(z, ids, top, lse, temperature, weight, z.dtype)
    alone = torch.full((n,), 55.0, device="cuda")
    pdb.pdb_distill(tok, z, ids, top, alone, teacher_lse=lse, temperature=temperature)
    N.assert_near(alone, want, tol, "loss")
    d = z if inplace else _lay(torch.full_like(z.contiguous(), 9.0), layout)
    loss = torch.full((n,), 55.0, device="cuda") if with_loss else None
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, weight=weight, dlogits=d, temperature=temperature)
    if with_loss:
        N.assert_near(loss, want, tol, "loss beside the gradient")
    N.assert_near(d, grad, tol_g, "dlogits")
    return alone, d


@pytest.mark.parametrize("kind", list(N.TYPES))
@pytest.mark.parametrize("bucket", [False, True])
@pytest.mark.parametrize("cols,K", [(1, 1), (2, 1), (9, 4), (33, 33), (300, 8), (1000, 64), (4099, 100), (32_000, 7),
                                    (50_001, 200), (131_073, 64)])
def test_loss_and_gradient(tok, kind, bucket, cols, K):
    g = _gen(cols + K)
    for n, layout, dl, T in [(1, "whole", "whole", 1.0), (5, "shifted", "shifted", 2.0), (2, "whole", "shifted", 0.5)]:
        z, ids, top, lse = _problem(n, cols, K, N.TYPES[kind], g, T, wide=n != 5)
        weight = torch.randn(n, device="cuda", generator=g)
        _check(tok, _lay(z, layout), ids, top, lse if bucket else None, T, weight, dl)
    z, ids, top, lse = _problem(3, cols, K, N.TYPES[kind], g)
    _check(tok, _lay(z, "shifted"), ids, top, lse if bucket else None, inplace=True, with_loss=False)
    pdb.check_tokens(tok)


@pytest.mark.parametrize("n,cols,K", [(500, 700, 16), (33, 20_000, 1024), (1, 300_000, 128), (3, 600_000, 50)])
def test_sizes(tok, n, cols, K):
    g = _gen(n)
    z, ids, top, lse = _problem(n, cols, K, torch.bfloat16, g, 1.5)
    _check(tok, z, ids, top, lse, 1.5, torch.rand(n, device="cuda", generator=g))
    _check(tok, z, ids, top, None, 1.5)


@pytest.mark.parametrize("top_type", list(N.TYPES))
def test_teacher_types(tok, top_type):
    g = _gen(21)
    z, ids, top, lse = _problem(6, 800, 12, torch.float32, g, top_type=N.TYPES[top_type], wide=False)
    wide = torch.zeros(6, 20, device="cuda").to(top.dtype)
    wide[:, 3:15] = top
    apart = torch.full((6, 17), 1 << 30, device="cuda", dtype=ids.dtype)
    apart[:, 2:14] = ids
    _check(tok, z, apart[:, 2:14], wide[:, 3:15], lse)         # rows of teacher logits and of ids with a stride
    _check(tok, z, ids, top, None)


@pytest.mark.parametrize("bucket", [False, True])
@pytest.mark.parametrize("cols", [40, 3000])
def test_empty_repeated_and_masked_slots(tok, bucket, cols):
    g = _gen(22)
    z, ids, top, lse = _problem(9, cols, 10, torch.float32, g)
    ids[0, 3:] = -1                                # three slots
    ids[1, :] = -1                                 # none
    ids[2, ::2] = -5
    ids[3, 4] = ids[3, 0]                          # a token twice, and three times
    ids[4, 1:4] = ids[4, 0]
    ids[5, :] = ids[5, 0]
    top[6, 5:] = -INF                              # slots that the teacher masks out
    top[7, :] = -INF
    top[1, 2] = NAN                                # in an empty slot: not looked at
    # repeated slots: the teacher's sum must stay below the whole
    t = torch.where(ids >= 0, top, -INF)
    t[1, 2] = -INF
    lse = torch.logaddexp(lse, torch.logsumexp(t, 1) + 0.1)
    loss, d = _check(tok, z, ids, top, lse if bucket else None)
    for r in (1, 7):
        assert float(loss[r]) == 0.0 and torch.count_nonzero(d[r]) == 0
    pdb.check_tokens(tok)


@pytest.mark.parametrize("bucket", [False, True])
def test_masked_students(tok, bucket):
    g = _gen(23)
    z, ids, top, lse = _problem(6, 2000, 8, torch.float32, g)
    z[0] = -INF                                    # nothing left: loss inf, gradient 0
    z[1, torch.rand(2000, device="cuda", generator=g) < 0.5] = -INF
    z[1, ids[1]] = 1.0                             # the slots stay
    z[2, ids[2, 3]] = -INF                         # the student rules out a slot: loss inf
    keep = torch.zeros(2000, dtype=torch.bool, device="cuda")
    keep[ids[3]] = True
    z[3, ~keep] = -INF                             # nothing outside of the slots
    z[4, ~keep] = torch.finfo(torch.float32).min
    loss, d = _check(tok, z, ids, top, lse if bucket else None)
    assert float(loss[0]) == INF and float(loss[2]) == INF and torch.count_nonzero(d[0]) == 0
    assert (float(loss[3]) == INF) == bucket


def test_weights_of_zero_shut_out_what_a_row_holds(tok):
    g = _gen(24)
    z, ids, top, lse = _problem(4, 500, 6, torch.bfloat16, g)
    z[1, 3], z[2, :] = NAN, INF
    weight = torch.tensor([1.0, 0.0, 0.0, 2.0], device="cuda")
    _, d = _check(tok, z, ids, top, lse, weight=weight)
    assert torch.count_nonzero(d[1:3]) == 0 and torch.isfinite(d).all()


def test_nan_in_a_row(tok):
    g = _gen(25)
    z, ids, top, lse = _problem(4, 500, 6, torch.float32, g)
    z[1, 3] = NAN
    top[2, 1] = NAN
    loss, d = torch.zeros(4, device="cuda"), torch.empty_like(z)
    for l in (None, lse):
        pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=l, dlogits=d)
        assert torch.isnan(loss).tolist() == [False, True, True, False]
        assert torch.isnan(d[1]).all() and torch.isnan(d[2, ids[2, 1]]) and torch.isfinite(d[[0, 3]]).all()


def test_a_student_surer_than_subtraction_can_tell(tok):
    # the student's probability outside of the slots is 1e-12: one minus the slots' sum in fp32 is rounding
    cols, K = 3000, 4
    z = torch.zeros(2, cols, device="cuda")
    ids = torch.tensor([[5, 9, 77, 2999], [0, 1, 2, 3]], device="cuda")
    z[0, ids[0]] = torch.tensor([36.0, 35.0, 34.0, 33.0], device="cuda")
    z[1, ids[1]] = torch.tensor([200.0, 201.0, 199.0, 198.0], device="cuda")       # e^-200: under fp32's range
    top = torch.tensor([[3.0, 2.0, 1.0, 0.0]] * 2, device="cuda")
    lse = torch.logsumexp(top, 1) + 0.05           # the teacher's rest is 5%
    loss, d = _check(tok, z, ids, top, lse)
    assert loss.min() > 1.0


def test_slots_out_of_range():
    g = _gen(26)
    for wide, beyond in ((False, 500), (True, (1 << 32) + 1)):
        tok = pdb.pdb_tokens_create()
        z, ids, top, lse = _problem(3, 500, 6, torch.float32, g, wide=wide)
        ids[1, 2] = -3
        _check(tok, z, ids, top, lse)
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_OK
        ids[1, 2] = beyond
        _check(tok, z, ids, top, lse)
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_ERANGE


@pytest.mark.parametrize("bucket", [False, True])
def test_gradient_against_differences(tok, bucket):
    # central differences of the definition in 64 bits; step h leaves h^2 / 6 of the third derivative
    # (T^2 w sums below 40 here) plus 64-bit rounding over h
    g = _gen(27)
    n, cols, K, T, step = 2, 13, 4, 1.5, 1e-4
    z, ids, top, lse = _problem(n, cols, K, torch.float32, g, T)
    ids[1, 2] = ids[1, 0]
    ids[1, 3] = -1
    if bucket:
        lse = lse + 0.5
    weight = torch.tensor([0.7, -1.3], device="cuda")
    (_, _), (_, tol) = N.distill(z, ids, top, lse if bucket else None, T, weight)
    d = torch.empty_like(z)
    pdb.pdb_distill(tok, z, ids, top, None, teacher_lse=lse if bucket else None, weight=weight, dlogits=d, temperature=T)
    i, t = ids.cpu(), top.double().cpu() / T
    used = i >= 0
    t = torch.where(used, t, -INF)
    lq = t - (lse.double().cpu() if bucket else torch.logsumexp(t, 1))[:, None]
    q = lq.exp()

    def value(x):
        lp = torch.log_softmax(x / T, 1)
        at = lp.gather(1, i.clamp(min=0))
        f = (q * (torch.where(used, lq, 0.0) - at)).sum(1)
        if bucket:
            inside = torch.zeros(n, cols + 1, dtype=torch.bool).scatter_(1, torch.where(used, i, cols), True)[:, :cols]
            rest = 1 - q.sum(1)
            f = f + rest * (rest.log() - torch.logsumexp(torch.where(inside, -INF, lp), 1))
        return (weight.double().cpu() * T * T * f).sum()
    x = z.double().cpu()
    for r in range(n):
        for j in range(cols):
            e = torch.zeros_like(x)
            e[r, j] = step
            diff = float((value(x + e) - value(x - e)) / (2 * step))
            assert abs(diff - float(d[r, j])) <= float(tol[r, j]) + 40 * step ** 2 + 1e-9


def test_loss_is_zero_where_student_and_teacher_agree(tok):
    g = _gen(28)
    z = torch.randn(5, 600, device="cuda", generator=g)
    top, ids = torch.topk(z, 10, dim=1)
    lse = torch.logsumexp(z, 1)
    loss, d = _check(tok, z, ids, top, lse)
    assert loss.abs().max() < 1e-5 and d.abs().max() < 1e-5


def test_same_bits_each_time(tok):
    g = _gen(29)
    z, ids, top, lse = _problem(30, 9000, 20, torch.bfloat16, g)
    a = _check(tok, z, ids, top, lse)
    b = _check(tok, z, ids, top, lse)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_on_another_stream():
    side = torch.cuda.Stream()
    big = torch.randn(8192, 8192, device="cuda")
    g = _gen(30)
    z, ids, top, lse = _problem(3, 4000, 5, torch.float32, g)
    given = z.clone()
    z.zero_()
    torch.cuda.synchronize()
    own = pdb.pdb_tokens_create()
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-4
        z.copy_(given)
        loss, d = torch.empty(3, device="cuda"), torch.empty_like(z)
        pdb.pdb_distill(own, z, ids, top, loss, teacher_lse=lse, dlogits=d)
    side.synchronize()
    (want, tol), (grad, tol_g) = N.distill(given, ids, top, lse, 1.0)
    N.assert_near(loss, want, tol, "loss")
    N.assert_near(d, grad, tol_g, "dlogits")


def test_refusals(tok):
    f = lambda *shape, **kw: torch.zeros(*shape, device="cuda", **kw)
    i = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int64)

    def refused(code, *a, **kw):
        with pytest.raises(pdb.PdbError) as e:
            pdb.pdb_distill(tok, *a, **kw)
        assert e.value.code == code, e.value
    z = f(4, 100)
    for a, kw in [((z, i(4, 5), f(4, 6), f(4)), {}), ((z, i(4, 5), f(3, 5), f(4)), {}), ((z, i(4, 5), f(4, 5), f(3)), {}),
                  ((z, i(4, 5), f(4, 5)), {}), ((z, i(4, 5), f(4, 5), f(4)), dict(temperature=0.0)),
                  ((z, i(4, 5), f(4, 5), f(4)), dict(temperature=INF)), ((z, i(4, 5), f(4, 5), f(4)), dict(dlogits=f(4, 99))),
                  ((z, i(4, 5), f(4, 5), f(4)), dict(dlogits=f(4, 100).half())),
                  ((z, i(4, 5), f(4, 5), f(4)), dict(weight=f(5), dlogits=f(4, 100))),
                  ((z, i(4, 5), f(4, 5), f(4)), dict(teacher_lse=f(4).double())),
                  ((z, f(4, 5), f(4, 5), f(4)), {}), ((z, i(4, 10)[:, ::2], f(4, 5), f(4)), {}), ((z, i(20), f(4, 5), f(4)), {}),
                  ((z, i(1, 5).expand(4, 5), f(4, 5), f(4)), {}),
                  ((z[:3], i(3, 5), f(3, 5), f(3)), dict(dlogits=z[1:]))]:
        refused(pdb.PDB_EINVAL, *a, **kw)
    refused(pdb.PDB_ETOOBIG, f(4, 2000), i(4, 1025), f(4, 1025), f(4))


def test_without_slots(tok):
    z, d = torch.ones(3, 50, device="cuda"), torch.ones(3, 50, device="cuda")
    loss = torch.ones(3, device="cuda")
    pdb.pdb_distill(tok, z, torch.zeros(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, 0, device="cuda"), loss,
                    dlogits=d)
    assert loss.tolist() == [0.0] * 3 and torch.count_nonzero(d) == 0


@pytest.mark.parametrize("n,cols,K,kind", [
    (1000, 10_200, 64, "bf16"), (700, 10_200, 65, "f16"), (700, 10_260, 64, "bf16"), (1300, 5100, 3, "f32"),   # 64 or 128 threads
    (300, 36_851, 9, "bf16"), (650, 36_871, 9, "f16"), (320, 73_702, 40, "bf16"),                              # one or two blocks
    (200, 36_877, 40, "f32"), (160, 73_720, 12, "f32"), (170, 73_741, 12, "f32")])                             # two or four
def test_rows_on_each_side_of_a_split(tok, n, cols, K, kind):
    # more rows than clusters at once, so that every cluster takes several; in place the same bits as beside
    g = _gen(cols + K)
    z, ids, top, lse = _problem(n, cols, K, N.TYPES[kind], g, 2.0)
    w = torch.rand(n, device="cuda", generator=g)
    w[1::7] = 0.0                                       # rows of zeros among the others
    ids[2::5, K // 2:] = -1                             # rows with empty slots
    loss, d = torch.full((n,), 55.0, device="cuda"), torch.full_like(z, 9.0)
    pdb.pdb_distill(tok, z, ids, top, loss, teacher_lse=lse, weight=w, dlogits=d, temperature=2.0)
    for rows in (slice(0, 6), slice(n // 2, n // 2 + 6), slice(n - 6, n)):
        (want, tol), (grad, tol_g) = N.distill(z[rows], ids[rows], top[rows], lse[rows], 2.0, w[rows], z.dtype)
        N.assert_near(loss[rows], want, tol, "loss")
        N.assert_near(d[rows], grad, tol_g, "dlogits")
    assert torch.count_nonzero(d[1::7]) == 0
    again = torch.full((n,), 55.0, device="cuda")
    pdb.pdb_distill(tok, z, ids, top, again, teacher_lse=lse, weight=w, dlogits=z, temperature=2.0)
    assert torch.equal(z, d) and torch.equal(again, loss)
    pdb.check_tokens(tok)
