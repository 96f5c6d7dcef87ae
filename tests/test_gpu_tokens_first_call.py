"""A process whose first call of an operator is recorded into a CUDA graph: what the library asks of the device once must not
disturb the recording."""
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

SCRIPT = """
import torch, paper_1508_00703_gb300 as pdb
z = torch.randn(700, 3000, device="cuda")
top, ids = torch.topk(z, 5, dim=1)
loss, d, want = torch.empty(700, device="cuda"), torch.empty_like(z), torch.empty_like(z)
lse, table = torch.empty(700, device="cuda"), torch.zeros(3000, 40, device="cuda")
tok = pdb.pdb_tokens_create(4000, 40)
some, rows = torch.randint(0, 3000, (4000,), device="cuda"), torch.ones(4000, 40, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    pdb.pdb_distill(tok, z, ids, top, loss, dlogits=d)
    pdb.pdb_logprobs(tok, z, lse=lse)
    pdb.pdb_embed_grad(tok, some, rows, table)
g.replay()
torch.cuda.synchronize()
other = torch.empty(700, device="cuda")
pdb.pdb_distill(tok, z, ids, top, other, dlogits=want)
pdb.check_tokens(tok)
assert torch.equal(loss, other) and torch.equal(d, want)
assert torch.allclose(lse, torch.logsumexp(z, 1), atol=1e-4)
assert torch.equal(table[:, 0], torch.bincount(some, minlength=3000).float())
print("recorded")
"""


def test_first_calls_recorded(repo_root):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    out = subprocess.run([sys.executable, "-c", SCRIPT], cwd=repo_root, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "recorded" in out.stdout, out.stderr[-2000:]
