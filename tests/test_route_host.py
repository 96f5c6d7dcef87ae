"""Argument checks of pdb_verify, pdb_route and its moves, and pdb_clip that need no GPU: every refusal comes before the first use of
a handle or of a pointer."""
import ctypes

import pytest

import paper_1508_00703_gb300 as pdb

F = 4096                                # an address that nothing reads


def _mat(rows, cols, stride=None, kind=pdb.PDB_TYPE_FLOAT, data=F):
    return pdb.pdb_mat(data, rows, cols, cols if stride is None else stride, kind)


@pytest.fixture(scope="module")
def lib():
    return pdb.load()


@pytest.fixture(scope="module")
def handle():
    # stands for a handle whose contents no refused call reads
    return ctypes.create_string_buffer(512)


BAD = [_mat(-1, 4), _mat(4, -1), _mat(4, 4, stride=3), _mat(4, 4, kind=3), _mat(4, 4, kind=-1), _mat(4, 4, data=None),
       _mat(4, 4, data=4098), _mat(4, 4, stride=1 << 60)]
FAR = dict(data=1 << 20)


def _verify(lib, handle, target=None, ids=pdb.pdb_ids(F, 2, 1, 0), D=1, draft=None, scale=1.0, draft_scale=1.0, u=F, v=F,
            tokens=F, accepted=F, logp=F):
    # two sequences of one draft
    return lib.pdb_verify(handle, _mat(4, 4) if target is None else target, ids, D, draft, scale, draft_scale, u, v, tokens,
                          accepted, logp, None)


def test_null_handles(lib):
    m = _mat(4, 4)
    assert _verify(lib, None) == pdb.PDB_EINVAL
    assert lib.pdb_route(None, pdb.pdb_ids(F, 8, 2, 0), 2, 4, 0, F, F, F, None) == pdb.PDB_EINVAL
    assert lib.pdb_route_rows(None, m, F, 1, F, _mat(4, 4, **FAR), None) == pdb.PDB_EINVAL
    assert lib.pdb_route_join(None, m, F, 1, F, _mat(4, 4, **FAR), None) == pdb.PDB_EINVAL
    assert lib.pdb_route_join_grad(None, m, F, 1, F, F, m, _mat(4, 4, **FAR), F, None) == pdb.PDB_EINVAL
    assert lib.pdb_clip(None, 1.0, 1.0, 0, F, None) == pdb.PDB_EINVAL
    lib.pdb_clip_plan_free(None)


@pytest.mark.parametrize("bad", range(len(BAD)))
def test_bad_matrices(lib, handle, bad):
    b, m = BAD[bad], _mat(4, 4, **FAR)
    h = ctypes.c_void_p(1)
    for rc in [_verify(lib, handle, target=b), _verify(lib, handle, draft=b),
               lib.pdb_route_rows(handle, b, F, 1, F, m, None), lib.pdb_route_rows(handle, m, F, 1, F, b, None),
               lib.pdb_route_join(handle, b, F, 1, F, m, None), lib.pdb_route_join(handle, m, F, 1, F, b, None),
               lib.pdb_route_join_grad(handle, b, F, 1, F, F, m, m, F, None),
               lib.pdb_route_join_grad(handle, m, F, 1, F, F, b, m, F, None),
               lib.pdb_route_join_grad(handle, m, F, 1, F, F, m, b, F, None),
               lib.pdb_clip_plan_build(b, m, 1, ctypes.byref(h), None), lib.pdb_clip_plan_build(m, b, 1, ctypes.byref(h), None)]:
        assert rc == pdb.PDB_EINVAL
    assert not h.value


def test_verify_refusals(lib, handle):
    for kw in (dict(target=_mat(3, 4)),                            # not whole sequences
               dict(target=_mat(4, 0)), dict(D=-1), dict(ids=None), dict(ids=pdb.pdb_ids(F, 3, 1, 0)),
               dict(ids=pdb.pdb_ids(None, 2, 1, 0)), dict(ids=pdb.pdb_ids(4100, 2, 1, 1)), dict(ids=pdb.pdb_ids(F, 2, 0, 0)),
               dict(draft=_mat(3, 4)), dict(draft=_mat(2, 5)), dict(draft=_mat(2, 4, kind=pdb.PDB_TYPE_HALF)),
               dict(u=None), dict(v=None), dict(tokens=None), dict(u=4097), dict(v=4098), dict(tokens=4097), dict(accepted=4097),
               dict(logp=4097)):
        assert _verify(lib, handle, **kw) == pdb.PDB_EINVAL, kw
    for x in (0.0, -1.0, float("inf"), float("nan"), 3e38):
        assert _verify(lib, handle, scale=x) == pdb.PDB_EINVAL
        assert _verify(lib, handle, draft=_mat(2, 4), draft_scale=x) == pdb.PDB_EINVAL
    assert _verify(lib, handle, target=_mat(4, (1 << 21) + 1)) == pdb.PDB_ETOOBIG
    assert _verify(lib, handle, target=_mat(66, 4), D=65, ids=pdb.pdb_ids(F, 65, 65, 0)) == pdb.PDB_ETOOBIG
    # no sequences: nothing to do
    none = pdb.pdb_mat(None, 0, 4, 4, 0)
    assert _verify(lib, handle, target=none, ids=pdb.pdb_ids(None, 0, 1, 0), u=None, v=None, tokens=None) == pdb.PDB_OK


def test_route_refusals(lib, handle):
    ids = pdb.pdb_ids(F, 8, 2, 0)
    for args in ((None, 2, 4, 0, F, F, F), (ids, 0, 4, 0, F, F, F), (ids, 3, 4, 0, F, F, F), (ids, 2, 0, 0, F, F, F),
                 (ids, 2, 4, -1, F, F, F), (ids, 2, 4, 0, None, F, F), (ids, 2, 4, 0, F, None, F), (ids, 2, 4, 0, F, F, None),
                 (ids, 2, 4, 0, 4097, F, F), (ids, 2, 4, 0, F, 4098, F), (ids, 2, 4, 0, F, F, 4099),
                 (pdb.pdb_ids(F, 8, 1, 0), 2, 4, 0, F, F, F), (pdb.pdb_ids(4100, 8, 2, 1), 2, 4, 0, F, F, F),
                 (pdb.pdb_ids(None, 8, 2, 0), 2, 4, 0, F, F, F), (pdb.pdb_ids(F, -2, 2, 0), 2, 4, 0, F, F, F)):
        assert lib.pdb_route(handle, *args, None) == pdb.PDB_EINVAL, args
    for args in ((pdb.pdb_ids(F, 130, 65, 0), 65, 4, 0), (ids, 2, 4097, 0), (ids, 2, 4, 1 << 30),
                 (pdb.pdb_ids(F, 1 << 32, 2, 0), 2, 4, 0)):
        assert lib.pdb_route(handle, *args, F, F, F, None) == pdb.PDB_ETOOBIG, args
    # the handle (zeros) has room for no slot
    assert lib.pdb_route(handle, ids, 2, 4, 0, F, F, F, None) == pdb.PDB_ETOOBIG


def test_move_refusals(lib, handle):
    m, far, n = _mat(4, 4), _mat(4, 4, **FAR), _mat(4, 4, data=1 << 24)
    rows, join, grad = lib.pdb_route_rows, lib.pdb_route_join, lib.pdb_route_join_grad
    for args in ((m, None, 1, F, far), (m, F, 0, F, far), (m, F, 1, None, far), (m, 4097, 1, F, far), (m, F, 1, 4098, far),
                 (m, F, 1, F, m), (m, F, 1, F, _mat(4, 5, **FAR))):
        assert rows(handle, *args, None) == pdb.PDB_EINVAL, args
    for args in ((m, None, 1, F, far), (m, F, 0, F, far), (m, F, 1, 4097, far), (m, F, 1, F, m), (m, F, 1, F, _mat(4, 5, **FAR))):
        assert join(handle, *args, None) == pdb.PDB_EINVAL, args
    for args in ((m, None, 1, F, F, far, n, F), (m, F, 0, F, F, far, n, F), (m, F, 1, None, F, far, n, F),
                 (m, F, 1, F, 4097, far, n, F), (m, F, 1, F, F, far, n, 4097), (None, F, 1, F, F, far, n, F),
                 (m, F, 1, F, F, far, n, None), (m, F, 1, F, F, far, far, F), (m, F, 1, F, F, _mat(4, 5, **FAR), n, F),
                 (_mat(5, 4), F, 1, F, F, far, n, F), (_mat(4, 4, kind=pdb.PDB_TYPE_HALF), F, 1, F, F, far, n, F),
                 (_mat(4, 4, data=(1 << 24) + 16), F, 1, F, F, far, n, F)):
        assert grad(handle, *args, None) == pdb.PDB_EINVAL, args
    assert rows(handle, m, F, 65, F, far, None) == pdb.PDB_ETOOBIG
    assert join(handle, m, F, 65, F, far, None) == pdb.PDB_ETOOBIG
    assert grad(handle, m, F, 65, F, F, far, n, F, None) == pdb.PDB_ETOOBIG
    wide = pdb.pdb_mat(F, 1 << 26, 1, 1, 0)
    assert join(handle, far, F, 64, F, wide, None) == pdb.PDB_ETOOBIG          # 2^32 slots
    # nothing to move
    assert rows(handle, _mat(0, 4, data=None), None, 1, None, _mat(0, 4, data=None), None) == pdb.PDB_OK
    assert join(handle, m, None, 1, None, _mat(0, 4, data=None), None) == pdb.PDB_OK
    assert grad(handle, None, None, 1, None, None, _mat(0, 4, data=None), _mat(0, 4, data=None), None, None) == pdb.PDB_OK


def _plan(lib, grads, outs, n=None):
    h = ctypes.c_void_p()
    g, o = (pdb.pdb_mat * len(grads))(*grads), (pdb.pdb_mat * len(outs))(*outs)
    rc = lib.pdb_clip_plan_build(g, o, len(grads) if n is None else n, ctypes.byref(h), None)
    assert not h.value
    return rc


def test_plan_refusals(lib):
    a, b = _mat(4, 4), _mat(4, 4, **FAR)
    assert lib.pdb_clip_plan_build(a, b, 1, None, None) == pdb.PDB_EINVAL
    h = ctypes.c_void_p()
    assert lib.pdb_clip_plan_build(None, b, 1, ctypes.byref(h), None) == pdb.PDB_EINVAL
    assert lib.pdb_clip_plan_build(a, None, 1, ctypes.byref(h), None) == pdb.PDB_EINVAL
    assert _plan(lib, [a], [b], -1) == pdb.PDB_EINVAL
    assert _plan(lib, [a], [_mat(4, 5, **FAR)]) == pdb.PDB_EINVAL
    assert _plan(lib, [a], [_mat(2, 8, **FAR)]) == pdb.PDB_EINVAL
    c = _mat(4, 4, data=1 << 24)
    assert _plan(lib, [a, c], [b, b]) == pdb.PDB_EINVAL                          # one result for two
    assert _plan(lib, [a, b], [b, c]) == pdb.PDB_EINVAL                          # a result over another's gradient
    assert _plan(lib, [a], [_mat(4, 4, data=F + 16)]) == pdb.PDB_EINVAL          # over its own, but not element for element
    assert _plan(lib, [a], [_mat(4, 4, data=F, kind=pdb.PDB_TYPE_HALF)]) == pdb.PDB_EINVAL
    x, y = _mat(4, 4, stride=8), _mat(4, 4, stride=8, data=F + 12)               # column ranges that share a column
    assert _plan(lib, [c, _mat(4, 4, data=1 << 26)], [x, y]) == pdb.PDB_EINVAL
    many = [_mat(1, 4, data=(1 << 24) + 64 * i) for i in range(300)]
    assert _plan(lib, [_mat(1, 4, data=(1 << 26) + 64 * i) for i in range(300)], many[:299] + [many[7]]) == pdb.PDB_EINVAL
    huge = _mat(1 << 30, 1 << 20), _mat(1 << 30, 1 << 20, data=1 << 60)
    assert _plan(lib, [huge[0]], [huge[1]]) == pdb.PDB_ETOOBIG


def test_clip_refusals(lib, handle):
    for bad in (-1.0, float("nan")):
        assert lib.pdb_clip(handle, bad, 1.0, 0, F, None) == pdb.PDB_EINVAL
    for bad in (float("inf"), float("nan")):
        assert lib.pdb_clip(handle, 1.0, bad, 0, F, None) == pdb.PDB_EINVAL
    assert lib.pdb_clip(handle, 1.0, 1.0, 0, 4097, None) == pdb.PDB_EINVAL
