"""A handle belongs to the device that was current at its creation: a call with another one current is refused before anything
is launched.  One device is enough to see it: the handle is told that it belongs to another."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu


def test_another_device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    tok = pdb.pdb_tokens_create(8, 4)
    z, ids = torch.zeros(3, 4, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    out, f = torch.full((3, 4), 7.0, device="cuda"), torch.full((3,), 7.0, device="cuda")
    slots = torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    calls = [lambda: pdb.pdb_embed(tok, z, ids, out), lambda: pdb.pdb_embed_grad(tok, ids, z, out),
             lambda: pdb.pdb_logprobs(tok, z, lse=f), lambda: pdb.pdb_logprobs_grad(tok, z, ids, f, None, f, None, out),
             lambda: pdb.pdb_distill(tok, z, slots, torch.zeros(3, 2, device="cuda"), f),
             lambda: pdb.pdb_distill(tok, z, slots, torch.zeros(3, 2, device="cuda"), f, dlogits=out)]
    device = ctypes.cast(tok.handle, ctypes.POINTER(ctypes.c_int))         # the handle's first member
    assert device[0] == torch.cuda.current_device()
    device[0] += 1
    try:
        for call in calls:
            with pytest.raises(pdb.PdbError) as e:
                call()
            assert e.value.code == pdb.PDB_EINVAL
        assert pdb.pdb_tokens_status(tok) == pdb.PDB_EINVAL
    finally:
        device[0] -= 1
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (f == 7.0).all()
    for call in calls:
        call()
    pdb.check_tokens(tok)
