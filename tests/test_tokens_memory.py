"""Where matrices of the token operators lie, as far as refusals show it without a GPU: matrices that share
memory are refused however their rows lie to one another, and so are extents that no memory holds."""
import ctypes
import random

import pytest

import paper_1508_00703_gb300 as pdb

BASE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return pdb.load()


@pytest.fixture(scope="module")
def handle():
    # stands for a handle whose contents no refused call reads
    return ctypes.create_string_buffer(512)


def _bytes(m):
    return 4 if m.type == pdb.PDB_TYPE_FLOAT else 2


def _meet(a, b):
    for i in range(a.rows):
        lo = a.data + i * a.stride * _bytes(a)
        for j in range(b.rows):
            at = b.data + j * b.stride * _bytes(b)
            if lo < at + b.cols * _bytes(b) and at < lo + a.cols * _bytes(a):
                return True
    return False


def test_shared_memory_is_refused(lib, handle):
    rng = random.Random(7)
    refused = 0
    while refused < 4000:
        kinds = [rng.choice([pdb.PDB_TYPE_FLOAT, pdb.PDB_TYPE_BFLOAT, pdb.PDB_TYPE_HALF]) for _ in range(2)]
        cols = rng.randrange(1, 7)
        rows = [rng.randrange(1, 6) for _ in range(2)]
        strides = [cols + rng.randrange(12) for _ in range(2)]
        if rng.random() < 0.5:
            strides[1], kinds[1] = strides[0], kinds[0]
        a, b = (pdb.pdb_mat(BASE + 4 * rng.randrange(80), rows[i], cols, strides[i], kinds[i]) for i in range(2))
        if not _meet(a, b):
            continue
        refused += 1
        ids = pdb.pdb_ids(4096, b.rows, 1, 0)
        assert lib.pdb_embed(handle, a, ids, 1.0, -1, b, None) == pdb.PDB_EINVAL
        assert lib.pdb_embed_grad(handle, ids, b, 1.0, -1, 0, a, None) == pdb.PDB_EINVAL


@pytest.mark.parametrize("rows,stride", [(2, (1 << 63) - 1), (5, 1 << 61), (1 << 30, 1 << 33), ((1 << 31) - 1, 1 << 40)])
def test_extents_past_any_memory(lib, handle, rows, stride):
    i, f = pdb.pdb_ids(4096, rows, 1, 0), 4096
    far, near = pdb.pdb_mat(BASE, rows, 4, stride, 0), pdb.pdb_mat(BASE, rows, 4, 4, 0)
    for rc in [lib.pdb_embed(handle, far, i, 1.0, -1, near, None), lib.pdb_embed(handle, near, i, 1.0, -1, far, None),
               lib.pdb_embed_grad(handle, i, far, 1.0, -1, 0, near, None),
               lib.pdb_logprobs(handle, far, i, 1.0, -100, f, f, f, 0, None, None, None),
               lib.pdb_logprobs_grad(handle, near, i, 1.0, -100, f, f, f, f, far, None),
               lib.pdb_distill(handle, near, pdb.pdb_ids(4096, rows * 4, 4, 0), far, None, 1.0, f, None, None, None)]:
        assert rc == pdb.PDB_EINVAL
    ids = pdb.pdb_ids(4096, rows, stride, 0)
    assert lib.pdb_logprobs(handle, near, ids, 1.0, -100, f, f, f, 0, None, None, None) == pdb.PDB_EINVAL
