"""Argument checks of the token operators that need no GPU: every refusal comes
before the first use of the handle or of a pointer."""
import ctypes

import pytest

import paper_1508_00703_gb300 as pdb


def _mat(rows, cols, stride=None, kind=pdb.PDB_TYPE_FLOAT, data=4096):
    return pdb.pdb_mat(data, rows, cols, cols if stride is None else stride, kind)


@pytest.fixture(scope="module")
def lib():
    return pdb.load()


@pytest.fixture(scope="module")
def handle():
    # stands for a handle whose contents no refused call reads
    return ctypes.create_string_buffer(512)


BAD = [_mat(-1, 4), _mat(4, -1), _mat(4, 4, stride=3), _mat(4, 4, kind=3), _mat(4, 4, kind=-1), _mat(4, 4, data=None),
       _mat(4, 4, data=4098)]


def test_null_handles(lib):
    m, i = _mat(4, 4), pdb.pdb_ids(4096, 4, 1, 0)
    h = ctypes.c_void_p()
    assert lib.pdb_tokens_create(4, 4, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_tokens_create(-1, 4, ctypes.byref(h), None) == pdb.PDB_EINVAL
    assert lib.pdb_tokens_create(1 << 31, 4, ctypes.byref(h), None) == pdb.PDB_ETOOBIG
    assert lib.pdb_tokens_status(None, None) == pdb.PDB_EINVAL
    lib.pdb_tokens_free(None)
    assert lib.pdb_embed(None, m, i, 1.0, -1, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_embed_grad(None, i, m, 1.0, -1, 0, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs(None, m, i, 1.0, -100, 4096, None, None, 0, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs_grad(None, m, i, 1.0, -100, 4096, 4096, 4096, 4096, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_distill(None, m, i, m, None, 1.0, 4096, None, None, None) == pdb.PDB_EINVAL


@pytest.mark.parametrize("bad", range(len(BAD)))
def test_bad_matrices(lib, handle, bad):
    b, m, i = BAD[bad], _mat(4, 4, data=1 << 20), pdb.pdb_ids(4096, 4, 1, 0)
    j = pdb.pdb_ids(4096, 16, 4, 0)
    f = 4096
    for rc in [lib.pdb_embed(handle, b, i, 1.0, -1, m, None), lib.pdb_embed(handle, m, i, 1.0, -1, b, None),
               lib.pdb_embed_grad(handle, i, b, 1.0, -1, 0, m, None),
               lib.pdb_embed_grad(handle, i, m, 1.0, -1, 0, b, None),
               lib.pdb_logprobs(handle, b, i, 1.0, -100, f, f, f, 0, None, None, None),
               lib.pdb_logprobs_grad(handle, b, i, 1.0, -100, f, f, f, f, m, None),
               lib.pdb_logprobs_grad(handle, m, i, 1.0, -100, f, f, f, f, b, None),
               lib.pdb_distill(handle, b, j, m, None, 1.0, f, None, None, None),
               lib.pdb_distill(handle, m, j, b, None, 1.0, f, None, None, None),
               lib.pdb_distill(handle, m, j, m, None, 1.0, f, None, b, None)]:
        assert rc == pdb.PDB_EINVAL


def test_null_matrices_and_ids(lib, handle):
    m, i, f = _mat(4, 4), pdb.pdb_ids(4096, 4, 1, 0), 4096
    assert lib.pdb_embed(handle, None, i, 1.0, -1, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_embed(handle, m, None, 1.0, -1, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_embed_grad(handle, None, m, 1.0, -1, 0, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs(handle, m, None, 1.0, -100, f, f, f, 0, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs(handle, None, None, 1.0, -100, None, f, f, 0, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs_grad(handle, m, None, 1.0, -100, f, f, f, f, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_distill(handle, m, None, m, None, 1.0, f, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_embed(handle, m, pdb.pdb_ids(4096, 4, 0, 0), 1.0, -1, _mat(4, 4, data=1 << 20), None) == pdb.PDB_EINVAL
    assert lib.pdb_distill(handle, m, pdb.pdb_ids(4096, 16, 3, 0), m, None, 1.0, f, None, None, None) == pdb.PDB_EINVAL
    odd = pdb.pdb_ids(4100, 4, 1, 1)                              # 64-bit ids at an odd word
    assert lib.pdb_embed(handle, m, odd, 1.0, -1, _mat(4, 4, data=1 << 20), None) == pdb.PDB_EINVAL


def test_bad_numbers(lib, handle):
    m, i, f = _mat(4, 4), pdb.pdb_ids(4096, 4, 1, 0), 4096
    j = pdb.pdb_ids(4096, 16, 4, 0)
    for x in (0.0, -1.0, float("inf"), float("nan")):
        assert lib.pdb_logprobs(handle, m, i, x, -100, f, f, f, 0, None, None, None) == pdb.PDB_EINVAL
        assert lib.pdb_logprobs_grad(handle, m, i, x, -100, f, f, f, f, m, None) == pdb.PDB_EINVAL
        assert lib.pdb_distill(handle, m, j, m, None, x, f, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs(handle, m, i, 1.0, -100, f, f, f, -1, f, f, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs(handle, m, i, 1.0, -100, f, f, f, 5, f, f, None) == pdb.PDB_EINVAL      # k > cols
    wide = _mat(4, 1000)
    assert lib.pdb_logprobs(handle, wide, i, 1.0, -100, f, f, f, 65, f, f, None) == pdb.PDB_ETOOBIG
    k = pdb.pdb_ids(4096, 4 * 1025, 1025, 0)
    assert lib.pdb_distill(handle, m, k, _mat(4, 1025), None, 1.0, f, None, None, None) == pdb.PDB_ETOOBIG
    assert lib.pdb_distill(handle, m, j, m, None, 1.0, None, None, None, None) == pdb.PDB_EINVAL    # nothing to write
    assert lib.pdb_logprobs_grad(handle, m, i, 1.0, -100, None, f, f, f, m, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs_grad(handle, m, i, 1.0, -100, f, None, f, f, m, None) == pdb.PDB_EINVAL


def test_results_over_their_inputs(lib, handle):
    # the logits' own memory is allowed only element for element
    i, f = pdb.pdb_ids(4096, 4, 1, 0), 4096
    j = pdb.pdb_ids(4096, 16, 4, 0)
    m = _mat(4, 4, stride=8, data=1 << 20)
    for d in (_mat(4, 4, stride=4, data=1 << 20), _mat(4, 4, stride=8, data=(1 << 20) + 4),
              _mat(4, 4, stride=8, data=(1 << 20) - 64)):
        assert lib.pdb_logprobs_grad(handle, m, i, 1.0, -100, f, f, f, f, d, None) == pdb.PDB_EINVAL
        assert lib.pdb_distill(handle, m, j, _mat(4, 4), None, 1.0, f, None, d, None) == pdb.PDB_EINVAL
    assert lib.pdb_embed(handle, m, i, 1.0, -1, m, None) == pdb.PDB_EINVAL
    for d in (_mat(4, 5), _mat(3, 4), _mat(4, 4, kind=pdb.PDB_TYPE_HALF)):
        assert lib.pdb_logprobs_grad(handle, m, i, 1.0, -100, f, f, f, f, d, None) == pdb.PDB_EINVAL


def test_calls_without_rows(lib, handle):
    none = pdb.pdb_mat(None, 0, 4, 4, 0)
    i = pdb.pdb_ids(None, 0, 1, 1)
    assert lib.pdb_embed(handle, _mat(4, 4), i, 1.0, -1, none, None) == pdb.PDB_OK
    assert lib.pdb_logprobs(handle, none, i, 1.0, -100, None, None, None, 0, None, None, None) == pdb.PDB_OK
    assert lib.pdb_logprobs_grad(handle, none, i, 1.0, -100, None, None, None, None, none, None) == pdb.PDB_OK
    assert lib.pdb_distill(handle, none, i, none, None, 1.0, 4096, None, None, None) == pdb.PDB_OK
