"""Tokens to experts and back against plain forms: places and moved rows equal, sums and gradients within bounds that follow from their
fp32 arithmetic (u = 2^-24; a chain of c products and sums is off by c u of the sum of magnitudes), halved units for 16-bit results."""
import math

import pytest

from tests._tokens import SLACK, TYPES, U, assert_near, rounding

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()


@pytest.fixture(scope="module")
def tok():
    return pdb.pdb_tokens_create(600_000, 0)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _want_places(ids, experts, capacity):
    e = ids.cpu().long().reshape(-1)
    n = e.numel()
    rows = experts * capacity if capacity else n
    place, source = torch.full((n,), -1, dtype=torch.int32), torch.full((rows,), -1, dtype=torch.int32)
    ends = torch.zeros(experts, dtype=torch.int32)
    e = torch.where((e >= 0) & (e < experts), e, experts)
    order = torch.sort(e, stable=True).indices
    count = torch.bincount(e, minlength=experts + 1)
    at = 0
    first = 0
    for x in range(experts):
        mine = order[at:at + int(count[x])]
        at += int(count[x])
        if capacity:
            first, mine = x * capacity, mine[:capacity]
        place[mine] = torch.arange(first, first + mine.numel(), dtype=torch.int32)
        source[first:first + mine.numel()] = mine.int()
        first += mine.numel()
        ends[x] = first
    return place.view(ids.shape), source, ends


def _route(tok, ids, experts, capacity=0):
    n, k = ids.shape
    place = torch.full((n, k), -9, device="cuda", dtype=torch.int32)
    source = torch.full((experts * capacity if capacity else n * k,), -9, device="cuda", dtype=torch.int32)
    ends = torch.full((experts,), -9, device="cuda", dtype=torch.int32)
    pdb.pdb_route(tok, ids, experts, place, source, ends, capacity=capacity)
    return place, source, ends


@pytest.mark.parametrize("n,k,experts", [(0, 1, 3), (1, 1, 1), (1, 8, 4096), (31, 2, 5), (255, 4, 8), (1024, 2, 64), (1025, 2, 1),
                                         (4096, 8, 60), (5000, 6, 256), (3000, 3, 1024), (2500, 7, 4000), (8192, 2, 60), (16_385, 1, 64), (65_536, 1, 4096), (65_537, 1, 128), (70_000, 8, 128),
                                         (9000, 64, 16)])
@pytest.mark.parametrize("capacity", [0, 1, 100])
@pytest.mark.parametrize("wide", [False, True])
def test_places(tok, n, k, experts, capacity, wide):
    g = _gen(n + k)
    # a few experts get most of the slots
    ids = (torch.rand(n, k, device="cuda", generator=g) ** 3 * experts).long().clamp(max=experts - 1)
    ids[torch.rand(n, k, device="cuda", generator=g) < 0.05] = -1
    ids = ids.to(torch.int64 if wide else torch.int32)
    for got, want in zip(_route(tok, ids, experts, capacity), _want_places(ids, experts, capacity)):
        assert torch.equal(got.cpu(), want)
    pdb.check_tokens(tok)


def test_one_expert_takes_all(tok):
    ids = torch.full((40_000, 2), 5, device="cuda", dtype=torch.int32)
    for capacity in (0, 1000):
        for got, want in zip(_route(tok, ids, 8, capacity), _want_places(ids, 8, capacity)):
            assert torch.equal(got.cpu(), want)
    nobody = torch.full((700, 2), -1, device="cuda", dtype=torch.int32)
    place, source, ends = _route(tok, nobody, 8)
    assert (place == -1).all() and (source == -1).all() and (ends == 0).all()


def test_ids_between_other_columns(tok):
    whole = torch.randint(-1, 9, (3000, 11), device="cuda", generator=_gen(1), dtype=torch.int32)
    for got, want in zip(_route(tok, whole[:, 2:6], 9), _want_places(whole[:, 2:6], 9, 0)):
        assert torch.equal(got.cpu(), want)


def test_ids_out_of_range():
    mine = pdb.pdb_tokens_create(6000, 0)
    ids = torch.randint(0, 9, (3000, 2), device="cuda", generator=_gen(1))
    ids[7, 1], ids[2999, 0] = 9, 1 << 40
    for got, want in zip(_route(mine, ids, 9), _want_places(ids, 9, 0)):
        assert torch.equal(got.cpu(), want)
    assert pdb.pdb_tokens_status(mine) == pdb.PDB_ERANGE
    with pytest.raises(pdb.PdbError) as e:
        _route(mine, torch.zeros(3001, 2, device="cuda", dtype=torch.int32), 9)
    assert e.value.code == pdb.PDB_ETOOBIG


def _plan(tok, n, k, experts, capacity, seed=0):
    g = _gen(seed)
    ids = torch.randint(-1, experts, (n, k), device="cuda", generator=g, dtype=torch.int32)
    return _route(tok, ids, experts, capacity)[:2]


def _matrix(rows, cols, dtype, g, layout):
    """Random values in a matrix of its own, or between other columns of a wider one, from any element on."""
    first, gap = layout
    whole = torch.full((rows, first + cols + gap), math.nan, device="cuda", dtype=dtype)
    m = whole[:, first:first + cols]
    m.copy_(torch.randn(rows, cols, device="cuda", generator=g))
    return m, whole


LAYOUTS = [(0, 0), (0, 8), (1, 2), (4, 4)]
SIZES = [(0, 2, 4, 0, 8), (1, 1, 1, 0, 1), (7, 2, 3, 0, 33), (40, 4, 8, 30, 8), (100, 8, 16, 0, 1000), (33, 3, 5, 9, 4104),
         (65, 64, 7, 0, 250), (300, 2, 4, 0, 2052), (5, 2, 64, 50, 516)]


@pytest.mark.parametrize("n,k,experts,capacity,dim", SIZES)
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16"), ("bf16", "f16")])
def test_rows(tok, n, k, experts, capacity, dim, a, b):
    place, source = _plan(tok, n, k, experts, capacity)
    for layout in LAYOUTS:
        x, _ = _matrix(n, dim, TYPES[a], _gen(2), layout)
        rows, whole = _matrix(source.numel(), dim, TYPES[b], _gen(3), layout)
        rows.fill_(math.nan)
        pdb.pdb_route_rows(tok, x, place, source, rows)
        want = torch.zeros(source.numel(), dim, device="cuda")
        used = source >= 0
        want[used] = x[(source[used] // k).long()].float()
        assert torch.equal(rows, want.to(rows.dtype))
        assert whole[:, :layout[0]].isnan().all() and whole[:, layout[0] + dim:].isnan().all()


@pytest.mark.parametrize("n,k,experts,capacity,dim", SIZES)
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("weighted", [False, True])
def test_join(tok, n, k, experts, capacity, dim, a, b, weighted):
    place, source = _plan(tok, n, k, experts, capacity)
    weight = torch.randn(n, k, device="cuda", generator=_gen(7)) if weighted else None
    for layout in LAYOUTS:
        rows, _ = _matrix(source.numel(), dim, TYPES[a], _gen(4), layout)
        rows[source < 0] = math.nan                           # read by nobody
        if weighted:
            weight[place < 0] = math.nan
        y, whole = _matrix(n, dim, TYPES[b], _gen(5), layout)
        pdb.pdb_route_join(tok, rows, place, y, weight=weight)
        there = (place >= 0)[:, :, None]
        v = torch.where(there, rows.double()[place.long().clamp(min=0)] if rows.numel() else
                        torch.zeros(n, k, dim, device="cuda", dtype=torch.float64), 0.0)
        if weighted:
            v = v * torch.where(there, weight.double()[:, :, None], 0.0)
        want = v.sum(1)
        assert_near(y, want, SLACK * U * (k + 1) * v.abs().sum(1) + rounding(want, y.dtype), "join")
        assert whole[:, :layout[0]].isnan().all() and whole[:, layout[0] + dim:].isnan().all()


@pytest.mark.parametrize("n,k,experts,capacity,dim", SIZES)
@pytest.mark.parametrize("a,b", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("form", ["all", "in place", "no weights", "rows alone"])
def test_join_grad(tok, n, k, experts, capacity, dim, a, b, form):
    place, source = _plan(tok, n, k, experts, capacity)
    there = (place >= 0)[:, :, None]
    at = place.long().clamp(min=0)
    for layout in LAYOUTS:
        rows, _ = _matrix(source.numel(), dim, TYPES[a], _gen(4), layout)
        dy, _ = _matrix(n, dim, TYPES[b], _gen(5), layout)
        weight = None if form == "no weights" else torch.randn(n, k, device="cuda", generator=_gen(7))
        w = torch.ones(n, k, device="cuda") if weight is None else weight
        v = rows.double()[at] if rows.numel() else torch.zeros(n, k, dim, device="cuda", dtype=torch.float64)
        part = torch.where(there, v * dy.double()[:, None], 0.0)
        want_w = part.sum(2)
        tol_w = SLACK * U * (dim / 32 + 45) * part.abs().sum(2)        # a lane's chain, its warp's five steps, eight warps
        want = torch.zeros(rows.shape, device="cuda", dtype=torch.float64)
        used = source >= 0
        slot = source[used].long()
        want[used] = w.double().view(-1)[slot, None] * dy.double()[slot // k]
        drows, whole = (rows, None) if form == "in place" else _matrix(source.numel(), dim, TYPES[a], _gen(6), layout)
        if form != "in place":
            drows.fill_(math.nan)
        dweight = None if form == "rows alone" else torch.full((n, k), math.nan, device="cuda")
        pdb.pdb_route_join_grad(tok, None if form == "rows alone" else rows, place, source, dy, drows, weight=weight, dweight=dweight)
        assert_near(drows, want, U * want.abs() + rounding(want, drows.dtype), "drows")
        if dweight is not None:
            assert_near(dweight, want_w, tol_w, "dweight")
        if whole is not None:
            assert whole[:, :layout[0]].isnan().all() and whole[:, layout[0] + dim:].isnan().all()


def test_gradients_by_differences(tok):
    # the whole way, tokens to rows to a weighted sum, is linear in each argument: differences of any size are its gradient
    n, k, experts, dim = 50, 3, 6, 40
    place, source = _plan(tok, n, k, experts, 0)
    g = _gen(9)
    x, dy, dx = (torch.randn(n, dim, device="cuda", generator=g) for _ in range(3))
    weight, dw = (torch.randn(n, k, device="cuda", generator=g) for _ in range(2))

    def loss(x, weight):
        rows, y = torch.empty(n * k, dim, device="cuda"), torch.empty(n, dim, device="cuda")
        pdb.pdb_route_rows(tok, x, place, source, rows)
        pdb.pdb_route_join(tok, rows, place, y, weight=weight)
        return float((y.double() * dy.double()).sum()), rows
    base, rows = loss(x, weight)
    drows, dweight, got = torch.empty_like(rows), torch.empty_like(weight), torch.empty_like(x)
    pdb.pdb_route_join_grad(tok, rows, place, source, dy, drows, weight=weight, dweight=dweight)
    pdb.pdb_route_join(tok, drows, place, got)
    # each loss: sums of k products, n dim of them of size about 4 k: k u of the magnitudes; the gradients alike
    size = float((weight.abs().sum(1)[:, None] * (x.abs() + dx.abs()) * dy.abs()).sum() + ((weight.abs() + dw.abs()).sum(1)[:, None] * x.abs() * dy.abs()).sum())
    tol = 4 * SLACK * U * (k + dim / 32 + 45) * size
    assert abs(loss(x + dx, weight)[0] - base - float((got.double() * dx.double()).sum())) < tol + U * size
    assert abs(loss(x, weight + dw)[0] - base - float((dweight.double() * dw.double()).sum())) < tol + U * size


def test_places_out_of_range():
    mine = pdb.pdb_tokens_create(64, 0)
    x = torch.ones(4, 16, device="cuda")
    place = torch.tensor([[0], [99], [2], [-3]], device="cuda", dtype=torch.int32)
    source = torch.tensor([0, -1, 2], device="cuda", dtype=torch.int32)
    rows = torch.full((3, 16), math.nan, device="cuda")
    pdb.pdb_route_rows(mine, x, place, source, rows)
    assert rows[:, 0].tolist() == [1.0, 0.0, 1.0] and pdb.pdb_tokens_status(mine) == pdb.PDB_ERANGE
    for call in ("join", "grad"):
        mine = pdb.pdb_tokens_create(64, 0)
        y, dw = torch.full((4, 16), math.nan, device="cuda"), torch.full((4, 1), math.nan, device="cuda")
        if call == "join":
            pdb.pdb_route_join(mine, rows, place, y)
            assert y[:, 3].tolist() == [1.0, 0.0, 1.0, 0.0]
        else:
            d = torch.full((3, 16), math.nan, device="cuda")
            pdb.pdb_route_join_grad(mine, rows, place, source, x, d, dweight=dw)
            assert d[:, 5].tolist() == [1.0, 0.0, 1.0] and dw.view(-1).tolist() == [16.0, 0.0, 16.0, 0.0]
        assert pdb.pdb_tokens_status(mine) == pdb.PDB_ERANGE


def test_same_bits_every_time(tok):
    place, source = _plan(tok, 3000, 4, 16, 0)
    g = _gen(3)
    rows, dy, w = torch.randn(12_000, 520, device="cuda", generator=g), torch.randn(3000, 520, device="cuda", generator=g), torch.randn(3000, 4, device="cuda", generator=g)
    seen = None
    for _ in range(3):
        y, d, dw = torch.empty_like(dy), torch.empty_like(rows), torch.empty_like(w)
        pdb.pdb_route_join(tok, rows, place, y, weight=w)
        pdb.pdb_route_join_grad(tok, rows, place, source, dy, d, weight=w, dweight=dw)
        if seen:
            assert all(torch.equal(a, b) for a, b in zip(seen, (y, d, dw)))
        seen = y, d, dw


def test_a_layer_in_a_graph(tok):
    # route, rows, one product for each expert, join, and back, as one recorded graph on inputs that change
    n, k, experts, dim, capacity = 500, 2, 8, 64, 160
    g = _gen(4)
    ids = torch.randint(0, experts, (n, k), device="cuda", generator=g, dtype=torch.int32)
    x, dy = torch.randn(n, dim, device="cuda", generator=g), torch.randn(n, dim, device="cuda", generator=g)
    W = torch.randn(experts, dim, dim, device="cuda", generator=g) / 8
    weight = torch.rand(n, k, device="cuda", generator=g)
    place, source, ends = (torch.empty(s, device="cuda", dtype=torch.int32) for s in ((n, k), experts * capacity, experts))
    rows, y, dw, dx = torch.empty(experts * capacity, dim, device="cuda"), torch.empty_like(x), torch.empty_like(weight), torch.empty_like(x)
    drows = torch.empty_like(rows)

    def layer():
        pdb.pdb_route(tok, ids, experts, place, source, ends, capacity=capacity)
        pdb.pdb_route_rows(tok, x, place, source, rows)
        out = torch.bmm(rows.view(experts, capacity, dim), W).view(-1, dim)
        pdb.pdb_route_join(tok, out, place, y, weight=weight)
        pdb.pdb_route_join_grad(tok, out, place, source, dy, drows, weight=weight, dweight=dw)
        din = torch.bmm(drows.view(experts, capacity, dim), W.transpose(1, 2)).view(-1, dim)
        pdb.pdb_route_join(tok, din, place, dx)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    ids.copy_(torch.randint(-1, experts, (n, k), device="cuda", generator=g, dtype=torch.int32))
    x.copy_(torch.randn(n, dim, device="cuda", generator=g))
    graph.replay()
    got = [t.clone() for t in (place, source, ends, rows, y, dw, dx)]
    layer()
    assert all(torch.equal(a, b) for a, b in zip(got, (place, source, ends, rows, y, dw, dx)))
    # against the plain layer with its gradients
    xs, ws = x.double().requires_grad_(), weight.double().requires_grad_()
    there = (place >= 0).double()
    e = ids.long().clamp(min=0)
    each = torch.einsum("nd,nkde->nke", xs, W.double()[e])
    out = (each * (ws * there)[:, :, None]).sum(1)
    gx, gw = torch.autograd.grad((out * dy.double()).sum(), (xs, ws))
    # the products in torch may round to tf32 where a program asks for that; here they are fp32: dim u of the magnitudes
    size = torch.einsum("nd,nkde->nke", x.double().abs(), W.double().abs()[e]).sum(1) * 2
    assert ((y.double() - out).abs() <= SLACK * U * (dim + k + 8) * size).all()
    assert ((dw.double() - gw).abs() <= SLACK * U * (2 * dim + 64) * (size * dy.double().abs()).sum(1, keepdim=True)).all()
    back = torch.einsum("ne,nkde->nd", dy.double().abs(), W.double().abs()[e])
    assert ((dx.double() - gx).abs() <= SLACK * U * (dim + k + 8) * back).all()


def test_refusals(tok):
    ids = torch.zeros(4, 2, device="cuda", dtype=torch.int32)
    place, source, ends = _route(tok, ids, 3)
    x, rows, w = torch.ones(4, 8, device="cuda"), torch.ones(8, 8, device="cuda"), torch.ones(4, 2, device="cuda")
    for call in (lambda: pdb.pdb_route(tok, ids.float(), 3, place, source, ends), lambda: pdb.pdb_route(tok, ids.view(-1), 3, place, source, ends),
                 lambda: pdb.pdb_route(tok, ids, 3, place.long(), source, ends), lambda: pdb.pdb_route(tok, ids, 3, place, source[:7], ends),
                 lambda: pdb.pdb_route(tok, ids, 3, place, source, ends, capacity=2), lambda: pdb.pdb_route(tok, ids, 4, place, source, ends),
                 lambda: pdb.pdb_route_rows(tok, x, place[:3], source, rows), lambda: pdb.pdb_route_rows(tok, x, place, source[:7], rows),
                 lambda: pdb.pdb_route_rows(tok, x, place.view(-1), source, rows), lambda: pdb.pdb_route_rows(tok, x, place, source, rows[:, :4]),
                 lambda: pdb.pdb_route_rows(tok, x, place, source.cpu(), rows), lambda: pdb.pdb_route_rows(tok, x, place.t(), source, rows),
                 lambda: pdb.pdb_route_join(tok, rows, place, x, weight=w[:, :1]), lambda: pdb.pdb_route_join(tok, rows, place, x[:3]),
                 lambda: pdb.pdb_route_join(tok, rows, place, rows[:4]), lambda: pdb.pdb_route_join(tok, rows.double(), place, x),
                 lambda: pdb.pdb_route_join_grad(tok, None, place, source, x, rows, dweight=w),
                 lambda: pdb.pdb_route_join_grad(tok, rows, place, source, x, rows.clone(), dweight=w.half()),
                 lambda: pdb.pdb_route_join_grad(tok, rows.half(), place, source, x, rows, dweight=w),
                 lambda: pdb.pdb_route_join_grad(tok, rows, place, source, rows[:4], rows, dweight=w)):
        with pytest.raises(pdb.PdbError):
            call()


@pytest.mark.parametrize("n,k,capacity", [(5000, 2, 0), (4000, 8, 900), (16_384, 4, 0), (16_384, 8, 2500)])
def test_places_in_a_graph(tok, n, k, capacity):
    # by one cluster of several blocks, and by two launches, beside calls of other sizes on the same handle
    experts = 48
    g = _gen(9)
    ids = torch.randint(-1, experts, (n, k), device="cuda", generator=g)
    place, source, ends = (torch.empty(s, device="cuda", dtype=torch.int32) for s in ((n, k), experts * capacity or n * k, experts))
    other = torch.randint(0, experts, (17_000, 4), device="cuda", generator=g)
    there = [torch.empty(s, device="cuda", dtype=torch.int32) for s in ((17_000, 4), 68_000, experts)]
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        pdb.pdb_route(tok, other, experts, *there)
        pdb.pdb_route(tok, ids, experts, place, source, ends, capacity=capacity)
        pdb.pdb_route(tok, other, experts, *there)
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(3):
        ids.copy_(torch.randint(-1, experts, (n, k), device="cuda", generator=g))
        for t in (place, source, ends):
            t.fill_(-7)
        graph.replay()
        assert all(torch.equal(a, b.cpu()) for a, b in zip(_want_places(ids, experts, capacity), (place, source, ends)))
        assert torch.equal(there[2], torch.bincount(other.view(-1), minlength=experts).cumsum(0).int())
