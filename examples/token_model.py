"""A small next-token model trained from a teacher with the library's token operators.

The student is a bag of context: the scaled rows of the last `context` tokens, averaged,
times an output matrix.  A step is what a program does that trains such a model:

  pdb_embed           the context tokens' rows (the reads of a step, Definition 3)
  h @ W.T             logits
  pdb_distill         loss against the teacher's top logits, the gradient written over the logits
  d @ W, d.T @ h      gradients of h and W
  pdb_embed_grad      the SGD step on the table, in place, each id's rows summed in a fixed order

and pdb_logprobs then scores held-out text: log probability of the tokens that followed,
the model's entropy, and how often the token is among its five most probable.

The text is synthetic: a random teacher of the same form, its tokens drawn from its
own distribution, so the student can learn all of it.

  python examples/token_model.py [--steps N] [--vocab V] [--dim D] [--tokens N]
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1508_00703_gb300 as pdb


class Model:
    def __init__(self, vocab, dim, context, tokens, seed, spread):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.context, self.scale = context, math.sqrt(dim)
        self.table = torch.randn(vocab, dim, device="cuda", generator=g) * spread / math.sqrt(dim)
        self.out = torch.randn(vocab, dim, device="cuda", generator=g) * spread / math.sqrt(dim)
        self.tok = pdb.pdb_tokens_create(tokens * context, dim)
        self.rows = torch.empty(tokens * context, dim, device="cuda")

    def hidden(self, ids):
        """Mean of the scaled rows of each example's context (n, context)."""
        rows = self.rows[: ids.numel()]
        pdb.pdb_embed(self.tok, self.table, ids.view(-1), rows, scale=self.scale)
        return rows.view(ids.shape[0], self.context, -1).mean(1)

    def logits(self, ids):
        h = self.hidden(ids)
        return h, h @ self.out.t()

    def step(self, ids, top_ids, top_logits, teacher_lse, temperature, eta):
        """One SGD step on the mean distillation loss; returns the examples' losses."""
        n = ids.shape[0]
        h, logits = self.logits(ids)
        loss = torch.empty(n, device="cuda")
        weight = torch.full((n,), 1.0 / n, device="cuda")
        pdb.pdb_distill(self.tok, logits, top_ids, top_logits, loss, teacher_lse=teacher_lse, weight=weight,
                        dlogits=logits, temperature=temperature)
        dh = logits @ self.out
        self.out -= eta * (logits.t() @ h)
        drows = (dh / self.context).repeat_interleave(self.context, 0)
        pdb.pdb_embed_grad(self.tok, ids.view(-1), drows, self.table, scale=-eta * self.scale, accumulate=True)
        return loss

    def score(self, ids, following, k=5):
        """Mean log probability of the following tokens, mean entropy, share of them among the k most probable."""
        _, logits = self.logits(ids)
        n = ids.shape[0]
        logp, entropy = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        top = torch.empty(n, k, device="cuda", dtype=torch.int32)
        pdb.pdb_logprobs(self.tok, logits, following, logp, entropy=entropy, top_ids=top)
        hit = (top == following[:, None]).any(1).float().mean()
        return float(logp.mean()), float(entropy.mean()), float(hit)


def train(steps=400, vocab=2000, dim=64, tokens=1024, context=4, slots=32, temperature=2.0, eta=16.0, seed=0, log=None):
    """Trains and returns (losses, score before, score after, the teacher's score)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher = Model(vocab, dim, context, tokens, seed + 1, 1.7)
    student = Model(vocab, dim, context, tokens, seed + 2, 0.7)
    weight = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -1.0

    def batch():
        # contexts of word-like ids, and the teacher's logits there
        ids = torch.multinomial(weight, tokens * context, replacement=True, generator=g).view(tokens, context)
        return ids, teacher.logits(ids)[1]
    held, held_logits = batch()
    following = torch.multinomial(torch.softmax(held_logits, 1), 1, generator=g).view(-1)
    best = teacher.score(held, following)
    before = student.score(held, following)
    losses = []
    for i in range(steps):
        ids, logits = batch()
        top_logits, top_ids = torch.topk(logits, slots, dim=1)
        lse = torch.logsumexp(logits / temperature, 1)
        loss = student.step(ids, top_ids, top_logits, lse, temperature, eta)
        if i % max(1, steps // 20) == 0 or i == steps - 1:
            losses.append(float(loss.mean()))
            if log:
                log(f"step {i}: loss {losses[-1]:.4f}")
    pdb.check_tokens(student.tok)
    return losses, before, student.score(held, following), best


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--vocab", type=int, default=2000)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=1024, help="examples of a step")
    a = ap.parse_args()
    _, before, after, best = train(a.steps, a.vocab, a.dim, a.tokens, log=print)
    for name, (logp, entropy, hit) in (("before", before), ("after", after), ("teacher", best)):
        print(f"{name:8s} log probability {logp:.3f}  entropy {entropy:.3f}  among the first five {hit:.3f}")


if __name__ == "__main__":
    main()
