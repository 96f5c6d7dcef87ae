"""The example's drafting: one context, more than the models are made for, and small runs from its command line."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pdb = pytest.importorskip("paper_1508_00703_gb300")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    pdb.load()
    torch.backends.cuda.matmul.allow_tf32 = False


@pytest.mark.parametrize("experts", [0, 4])
@pytest.mark.parametrize("n", [1, 12, 13, 40, 70])
def test_any_number_of_contexts(experts, n):
    from examples import token_model as tm
    tokens, V, context = 64, 200, 3
    target = tm.Model(V, 16, context, tokens, 1, 1.7)
    draft = tm.Mixed(V, 16, context, tokens, 2, 1.0, experts) if experts else tm.Model(V, 16, context, tokens, 2, 1.0)
    ids = torch.randint(0, V, (n, context), device="cuda")
    text, accepted = tm.speculate(target, draft, ids, rounds=2)
    assert text.shape == (n, 2, 5) and accepted.shape == (n, 2)
    assert torch.equal((text >= 0).sum(2), accepted.long() + 1) and int(text.max()) < V
    # in slices as at once
    wide = tm.Model(V, 16, context, 400, 1, 1.7)
    every = torch.randint(0, V, (n * 5, context), device="cuda")
    assert torch.allclose(tm._logits(target, every), wide.logits(every)[1], rtol=1e-5, atol=1e-5)
    if experts:
        pdb.check_tokens(draft.experts.tok)


@pytest.mark.parametrize("args", [["--tokens", "64"], ["--tokens", "40", "--experts", "4"]])
def test_small_runs(args):
    done = subprocess.run([sys.executable, os.path.join("examples", "token_model.py"), "--steps", "2", "--vocab", "120", "--dim", "16", *args],
                          cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr[-2000:]
    assert "drafts accepted a round" in done.stdout
