"""pdb_clip against the formulas in 64 bits.  A thread adds at most 72 squares in fp32 one after the other (a piece of 16,384 elements and
7 more, by 256 threads) before the sums go on in 64 bits, so the sum of squares is off by 72 u of itself (u = 2^-24), the norm by half
of that and its rounding, and a step by that, the factor's rounding, two more, and its type's."""
import math

import pytest

from tests._tokens import TYPES, U, assert_near, rounding

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu
REL = 36 * U                            # of the norm in 64 bits


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _norm(grads):
    return math.sqrt(sum(float(d.double().square().sum()) for d in grads))


def _check(grads, outs, max_norm, scale, accumulate, plan=None, norm=None):
    s = float(torch.tensor(scale, dtype=torch.float32))
    N = _norm(grads)
    f = max_norm / N if N > max_norm else 1.0
    want, tol = [], []
    for d, o in zip(grads, outs):
        v = s * f * d.double()
        w = o.double() + v if accumulate else v
        want.append(w.cpu())
        tol.append(((REL + 4 * U) * v.abs() + (U * w.abs() if accumulate else 0.0) + rounding(w, o.dtype)).cpu())
    norm = torch.full((1,), -1.0, device="cuda") if norm is None else norm
    pdb.pdb_clip(pdb.pdb_clip_plan_build(grads, outs) if plan is None else plan, max_norm, norm, scale=scale, accumulate=accumulate)
    assert abs(float(norm) - N) <= (REL + U) * N + 2.0 ** -149, (float(norm), N)
    for i, (o, w, t) in enumerate(zip(outs, want, tol)):
        assert_near(o, w, t, f"result {i}")


SHAPES = [[(1,)], [()], [(5, 7)], [(0, 4), (3, 0), (9,)], [(1000, 33), (33,), (1,), (64, 64), (2, 3, 5)],
          [(300_001,)], [(2048, 520), (520,), (520,), (4097, 65)], [(1, 40_000)] + [(17,)] * 400]


@pytest.mark.parametrize("shapes", range(len(SHAPES)))
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16"), ("f16", "bf16")])
@pytest.mark.parametrize("max_norm,scale,accumulate", [(0.5, -0.1, True), (1e9, 1.0, False), (0.01, 2.0, False), (math.inf, 1.0, True)])
def test_steps(shapes, a, b, max_norm, scale, accumulate):
    g = _gen(shapes)
    grads = [torch.randn(s, device="cuda", generator=g).to(TYPES[a]) for s in SHAPES[shapes]]
    outs = [torch.randn(s, device="cuda", generator=g).to(TYPES[b]) for s in SHAPES[shapes]]
    _check(grads, outs, max_norm, scale, accumulate)


def test_no_gradients():
    norm = torch.full((1,), 5.0, device="cuda")
    pdb.pdb_clip(pdb.pdb_clip_plan_build([]), 1.0, norm)
    assert float(norm) == 0.0
    zero = torch.zeros(70, 9, device="cuda")
    pdb.pdb_clip(pdb.pdb_clip_plan_build([zero]), 0.0, norm)
    assert float(norm) == 0.0 and (zero == 0).all()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("first,gap", [(0, 0), (1, 0), (3, 5), (8, 8), (4, 0)])
def test_layouts(kind, first, gap):
    # gradients and results that start at any element, and column ranges of wider matrices
    g = _gen(first)
    rows, cols = 37, 1003
    whole = torch.full((rows, first + 2 * cols + gap), math.nan, device="cuda", dtype=TYPES[kind])
    d, o = whole[:, first:first + cols], whole[:, first + cols + gap:]
    d.copy_(torch.randn(rows, cols, device="cuda", generator=g))
    o.copy_(torch.randn(rows, cols, device="cuda", generator=g))
    flat = torch.randn(first + 20_000, device="cuda", generator=g).to(TYPES[kind])
    out = torch.full((gap + 20_000 + 1,), math.nan, device="cuda")
    kept = whole.clone()
    _check([d, flat[first:]], [o, out[gap:gap + 20_000]], 1.0, 1.0, False)
    rest = torch.ones(whole.shape[1], dtype=torch.bool)
    rest[first + cols + gap:] = False
    assert torch.equal(torch.nan_to_num(whole[:, rest]), torch.nan_to_num(kept[:, rest]))
    assert out[:gap].isnan().all() and out[-1].isnan()


@pytest.mark.parametrize("kind", list(TYPES))
def test_in_place(kind):
    g = _gen(2)
    grads = [torch.randn(s, device="cuda", generator=g).to(TYPES[kind]) for s in ((500, 77), (12_345,), (3,))]
    kept = [d.clone() for d in grads]
    plan, norm = pdb.pdb_clip_plan_build(grads), torch.empty(1, device="cuda")
    pdb.pdb_clip(plan, 1e6, norm)                            # not clipped: nothing changes
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    _check(kept, [torch.empty_like(d) for d in kept], 1.0, 1.0, False, norm=norm)
    pdb.pdb_clip(plan, 1.0, norm)
    apart = [torch.empty_like(d) for d in kept]
    pdb.pdb_clip(pdb.pdb_clip_plan_build(kept, apart), 1.0)
    assert all(torch.equal(a, b) for a, b in zip(grads, apart))
    pdb.pdb_clip(plan, math.inf, norm, scale=0.5)
    assert all(torch.equal(a, (b.float() * 0.5).to(b.dtype)) for a, b in zip(grads, apart))


@pytest.mark.parametrize("size", [1e30, 3e38, 1e-25, 1e-38, 1e-42])
def test_squares_outside_of_fp32(size):
    # some pieces' squares leave fp32's range at its top or bottom, others do not
    g = _gen(5)
    far = (torch.rand(3, 50_001, device="cuda", generator=g) + 0.1).clamp(max=1.0) * size
    far[1] = 0.0
    grads = [far, torch.zeros(40_000, device="cuda"), torch.full((9,), size, device="cuda")]
    outs = [torch.zeros_like(d) for d in grads]
    plan, norm = pdb.pdb_clip_plan_build(grads, outs), torch.empty(1, device="cuda")
    pdb.pdb_clip(plan, 1.0, norm, accumulate=True)
    N = _norm(grads)
    if N > torch.finfo(torch.float32).max:
        assert float(norm) == math.inf                       # rounded so; the step is formed from the norm itself
    else:
        assert abs(float(norm) - N) <= (REL + U) * N + 2.0 ** -149
    f = min(1.0, 1.0 / N)
    for d, o in zip(grads, outs):
        want = d.double() * f
        # a factor below fp32's normal range is off by half of its smallest step
        assert_near(o, want, (REL + 4 * U) * want.abs() + 2.0 ** -150 * d.double().abs() + 2.0 ** -149, "step")


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kind", list(TYPES))
def test_not_finite(bad, kind):
    g = _gen(6)
    for accumulate in (False, True):
        grads = [torch.randn(s, device="cuda", generator=g).to(TYPES[kind]) for s in ((100, 65), (70_000,))]
        grads[1][33_333] = bad
        outs = [torch.randn(d.shape, device="cuda", generator=g) for d in grads]
        kept, norm = [o.clone() for o in outs], torch.empty(1, device="cuda")
        pdb.pdb_clip(pdb.pdb_clip_plan_build(grads, outs), 1.0, norm, scale=-0.1, accumulate=accumulate)
        assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
        assert all(torch.equal(a, b) for a, b in zip(outs, kept))


def test_same_bits_every_time_and_in_graphs():
    g = _gen(7)
    grads = [torch.randn(s, device="cuda", generator=g) for s in ((4000, 300), (300,), (7, 11))]
    outs = [torch.zeros_like(d) for d in grads]
    plan, norm = pdb.pdb_clip_plan_build(grads, outs), torch.empty(1, device="cuda")
    pdb.pdb_clip(plan, 1.0, norm)
    first = [norm.clone()] + [o.clone() for o in outs]
    other = pdb.pdb_clip_plan_build(grads, [torch.zeros_like(d) for d in grads])
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pdb.pdb_clip(plan, 1.0, norm)
    with torch.cuda.graph(second):
        pdb.pdb_clip(plan, 0.5, None, scale=2.0)
    for o in outs:
        o.fill_(math.nan)
    graph.replay()
    second.replay()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip([norm] + outs, first))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pdb.pdb_clip(other, 1.0, norm)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip([norm] + other.tensors[1], first))
    # new gradients in the same memory
    for d in grads:
        d.copy_(torch.randn(d.shape, device="cuda", generator=g))
    _check(grads, outs, 1.0, 1.0, False, plan=plan)


def test_more_than_2_31_elements():
    # offsets past 32 bits: gradients of 2^31 + elements in 16 bits
    d = torch.full((1 << 16, (1 << 15) + 8), 2.0 ** -10, device="cuda", dtype=torch.bfloat16)
    norm = torch.empty(1, device="cuda")
    pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), 1.0, norm)
    N = math.sqrt(d.numel()) * 2.0 ** -10
    assert abs(float(norm) - N) <= (REL + U) * N
    want = float(torch.tensor(2.0 ** -10 / N).bfloat16())
    assert (d[0].float() == want).all() and (d[-1].float() == want).all() and (d[40_000].float() == want).all()


def test_refusals():
    d, o = torch.ones(4, 8, device="cuda"), torch.ones(4, 8, device="cuda")
    for call in (lambda: pdb.pdb_clip_plan_build([d], []), lambda: pdb.pdb_clip_plan_build([d], [o[:, :4]]),
                 lambda: pdb.pdb_clip_plan_build([d.double()]), lambda: pdb.pdb_clip_plan_build([d.cpu()]),
                 lambda: pdb.pdb_clip_plan_build([d.t()]), lambda: pdb.pdb_clip_plan_build([d, o], [o, d]),
                 lambda: pdb.pdb_clip_plan_build([d, d]), lambda: pdb.pdb_clip_plan_build([d], [o.view(8, 4)]),
                 lambda: pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), -1.0), lambda: pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), math.nan),
                 lambda: pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), 1.0, torch.empty(2, device="cuda")),
                 lambda: pdb.pdb_clip(pdb.pdb_clip_plan_build([d]), 1.0, scale=math.inf)):
        with pytest.raises(pdb.PdbError):
            call()
