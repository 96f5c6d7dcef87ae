"""Scales and temperatures whose factor leaves fp32's range are refused, without a GPU: 0 times an infinite factor would
make the row's own maximum a NaN."""
import ctypes

import pytest

import paper_1508_00703_gb300 as pdb


@pytest.fixture(scope="module")
def lib():
    return pdb.load()


@pytest.fixture(scope="module")
def handle():
    # stands for a handle whose contents no refused call reads
    return ctypes.create_string_buffer(512)


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales(lib, handle, scale):
    m, i, f = pdb.pdb_mat(1 << 20, 4, 4, 4, 0), pdb.pdb_ids(4096, 4, 1, 0), 4096
    d = pdb.pdb_mat(1 << 21, 4, 4, 4, 0)
    assert lib.pdb_logprobs(handle, m, i, scale, -100, f, f, f, 0, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_logprobs_grad(handle, m, i, scale, -100, f, f, f, f, d, None) == pdb.PDB_EINVAL


@pytest.mark.parametrize("temperature", [1e-45, 4e-39, 1.9e19, 3e38])
def test_temperatures(lib, handle, temperature):
    m, j, f = pdb.pdb_mat(1 << 20, 4, 4, 4, 0), pdb.pdb_ids(4096, 16, 4, 0), 4096
    d = pdb.pdb_mat(1 << 21, 4, 4, 4, 0)
    assert lib.pdb_distill(handle, m, j, m, None, temperature, f, None, None, None) == pdb.PDB_EINVAL
    assert lib.pdb_distill(handle, m, j, m, None, temperature, f, None, d, None) == pdb.PDB_EINVAL
