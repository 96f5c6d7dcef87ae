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

With experts (--experts E) the student has a layer of small matrices of which each example uses two, and its steps are clipped:

  pdb_route, pdb_route_rows     the examples' hidden rows to their experts, whose products are one batched one
  pdb_route_join                back, weighted by the router's probabilities (pdb_logprobs' alternatives)
  pdb_route_join_grad           the gradients of rows and weights
  pdb_clip                      the SGD step on all parameters, clipped to a norm over all gradients

At the end the student drafts for the teacher (pdb_verify): it proposes tokens, each drawn from its own distribution, the teacher
looks at all of them at once, and those that stay, with one more of its own, are distributed as the teacher's.

The text is synthetic: a random teacher of the same form, its tokens drawn from its
own distribution, so the student can learn all of it.

  python examples/token_model.py [--steps N] [--vocab V] [--dim D] [--tokens N] [--experts E]
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
        self.context, self.tokens, self.scale = context, tokens, math.sqrt(dim)
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


class Experts:
    """y[i] = h[i] + the sum over the example's `slots` most probable experts e of p_e(i) W_e h[i], p = softmax(R h); the rows of an expert
    stand together, `capacity` of them at most, so that the products of all are one."""

    def __init__(self, experts, dim, tokens, seed, slots=2):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.k, self.n = slots, experts
        self.capacity = -(-2 * slots * tokens // experts)
        self.W = torch.randn(experts, dim, dim, device="cuda", generator=g) * 0.1 / math.sqrt(dim)
        self.R = torch.randn(experts, dim, device="cuda", generator=g) / math.sqrt(dim)
        self.tok = pdb.pdb_tokens_create(tokens * slots, 0)

    def forward(self, h):
        n, dim = h.shape
        rows = self.n * self.capacity
        scores = h @ self.R.t()
        logp, ids = torch.empty(n, self.k, device="cuda"), torch.empty(n, self.k, device="cuda", dtype=torch.int32)
        pdb.pdb_logprobs(self.tok, scores, top_logp=logp, top_ids=ids)
        place, source, ends = (torch.empty(s, device="cuda", dtype=torch.int32) for s in ((n, self.k), rows, self.n))
        pdb.pdb_route(self.tok, ids, self.n, place, source, ends, capacity=self.capacity)
        x, y = torch.empty(rows, dim, device="cuda"), torch.empty_like(h)
        pdb.pdb_route_rows(self.tok, h, place, source, x)
        out = torch.bmm(x.view(self.n, self.capacity, dim), self.W.transpose(1, 2)).view(rows, dim)
        weight = logp.exp()
        pdb.pdb_route_join(self.tok, out, place, y, weight=weight)
        self.kept = h, scores, ids, place, source, x, out, weight
        return h + y

    def backward(self, dy, dW, dR):
        """Writes the gradients of W and R and returns that of h."""
        h, scores, ids, place, source, x, out, weight = self.kept
        dout, dweight, dh = torch.empty_like(out), torch.empty_like(weight), torch.empty_like(h)
        pdb.pdb_route_join_grad(self.tok, out, place, source, dy, dout, weight=weight, dweight=dweight)
        dout = dout.view(self.n, self.capacity, -1)
        torch.bmm(dout.transpose(1, 2), x.view(self.n, self.capacity, -1), out=dW)
        pdb.pdb_route_join(self.tok, torch.bmm(dout, self.W).view(x.shape), place, dh)
        # p_e of a chosen expert with respect to all scores: p_e ([e = f] - p_f)
        g = dweight * weight
        dscores = torch.softmax(scores, 1) * -g.sum(1, keepdim=True)
        dscores.scatter_add_(1, ids.long(), g)
        torch.mm(dscores.t(), h, out=dR)
        return dy + dh + dscores @ self.R


class Mixed(Model):
    """The model with a layer of experts behind the mean of its rows, trained by clipped steps."""

    def __init__(self, vocab, dim, context, tokens, seed, spread, experts, max_norm=1.0):
        super().__init__(vocab, dim, context, tokens, seed, spread)
        self.experts = Experts(experts, dim, tokens, seed + 7)
        self.max_norm, self.norm = max_norm, torch.empty(1, device="cuda")
        weights = [self.table, self.out, self.experts.W, self.experts.R]
        self.grads = [torch.zeros_like(w) for w in weights]
        self.plan = pdb.pdb_clip_plan_build(self.grads, weights)

    def logits(self, ids):
        h = self.experts.forward(self.hidden(ids))
        return h, h @ self.out.t()

    def gradients(self, ids, top_ids, top_logits, teacher_lse, temperature):
        """The examples' losses; the gradients of their mean are left in self.grads."""
        n = ids.shape[0]
        h, logits = self.logits(ids)
        loss = torch.empty(n, device="cuda")
        weight = torch.full((n,), 1.0 / n, device="cuda")
        pdb.pdb_distill(self.tok, logits, top_ids, top_logits, loss, teacher_lse=teacher_lse, weight=weight,
                        dlogits=logits, temperature=temperature)
        dtable, dout, dW, dR = self.grads
        torch.mm(logits.t(), h, out=dout)
        dh = self.experts.backward(logits @ self.out, dW, dR)
        drows = (dh / self.context).repeat_interleave(self.context, 0)
        pdb.pdb_embed_grad(self.tok, ids.view(-1), drows, dtable, scale=self.scale)
        return loss

    def step(self, ids, top_ids, top_logits, teacher_lse, temperature, eta):
        loss = self.gradients(ids, top_ids, top_logits, teacher_lse, temperature)
        pdb.pdb_clip(self.plan, self.max_norm, self.norm, scale=-eta, accumulate=True)
        return loss


def _logits(model, ids):
    """The logits behind any number of contexts, as many at a time as the model is made for."""
    parts = [model.logits(part)[1] for part in ids.split(model.tokens)]
    return parts[0] if len(parts) == 1 else torch.cat(parts)


def speculate(target, draft, ids, rounds=8, drafts=4, seed=0):
    """Text behind the contexts ids (n, context), `rounds` rounds of up to drafts + 1 tokens, distributed as the target's: the
    tokens (n, rounds, drafts + 1), -1 behind a round's last, and the number of accepted drafts (n, rounds)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, context = ids.shape
    tok, nothing = target.tok, torch.empty(n, 0, device="cuda")
    text, counts = [], []
    for _ in range(rounds):
        seq = torch.cat([ids, torch.zeros(n, drafts, device="cuda", dtype=ids.dtype)], 1)
        rows, drawn = [], torch.empty(n, 1, device="cuda", dtype=torch.int32)
        for d in range(drafts):
            rows.append(_logits(draft, seq[:, d:d + context].contiguous()))
            pdb.pdb_verify(tok, rows[-1], nothing.int(), nothing, torch.rand(n, device="cuda", generator=g), drawn)
            seq[:, context + d] = drawn[:, 0]
        every = seq.unfold(1, context, 1).reshape(-1, context).contiguous()      # (of one sequence it is a view)
        z = _logits(target, every)
        y = torch.stack(rows, 1).view(n * drafts, -1)
        tokens, accepted = torch.empty(n, drafts + 1, device="cuda", dtype=torch.int32), torch.empty(n, device="cuda", dtype=torch.int32)
        pdb.pdb_verify(tok, z, seq[:, context:], torch.rand(n, drafts, device="cuda", generator=g),
                       torch.rand(n, device="cuda", generator=g), tokens, accepted, draft=y)
        behind = torch.cat([ids, tokens.to(ids.dtype)], 1)
        ids = behind.gather(1, accepted.long()[:, None] + 1 + torch.arange(context, device="cuda"))
        text.append(tokens)
        counts.append(accepted)
    pdb.check_tokens(tok)
    return torch.stack(text, 1), torch.stack(counts, 1)


def train(steps=400, vocab=2000, dim=64, tokens=1024, context=4, slots=32, temperature=2.0, eta=16.0, seed=0, log=None,
          experts=0, models=None):
    """Trains and returns (losses, score before, score after, the teacher's score); the models go to the list `models`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    teacher = Model(vocab, dim, context, tokens, seed + 1, 1.7)
    student = Mixed(vocab, dim, context, tokens, seed + 2, 0.7, experts) if experts else \
        Model(vocab, dim, context, tokens, seed + 2, 0.7)
    if models is not None:
        models += [teacher, student]
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
    ap.add_argument("--experts", type=int, default=0, help="experts of the student (0: none)")
    a = ap.parse_args()
    models = []
    _, before, after, best = train(a.steps, a.vocab, a.dim, a.tokens, log=print, experts=a.experts, models=models)
    for name, (logp, entropy, hit) in (("before", before), ("after", after), ("teacher", best)):
        print(f"{name:8s} log probability {logp:.3f}  entropy {entropy:.3f}  among the first five {hit:.3f}")
    ids = torch.randint(0, a.vocab, (64, models[0].context), device="cuda")
    text, accepted = speculate(models[0], models[1], ids)
    print(f"drafting for the teacher: {float(accepted.float().mean()):.2f} of 4 drafts accepted a round, "
          f"{float((text >= 0).sum(2).float().mean()):.2f} tokens")


if __name__ == "__main__":
    main()
