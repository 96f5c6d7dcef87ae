"""The token operators, as a program that trains and serves a token model calls them, and their plain forms.

  op        embed          rows of a table by token id, scaled (forward)
            embed_grad     the table's gradient from the rows' gradients, every row of the table written
            embed_update   the same sum as an SGD step on the table in place
            logprobs       log probabilities of given tokens, entropy, the k most probable alternatives
            logprobs_train the same without alternatives, then the gradient with respect to the logits
            distill        loss against a teacher's top logits (forward), with its gradient when `grad`

  ids are Zipf distributed (exponent s) over a random permutation of the vocabulary.  Logits are a broad noise with a few
  raised tokens per row; `masked` is the share of tokens that a constrained decoder has set to -inf.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name=None, **kw):
    c = dict(op="embed", n=1, vocab=10_000, dim=0, type="bf16", out="bf16", s=1.0, wide=False, k=0, masked=0.0, grad=False,
             bucket=False, temperature=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decoding step of eight sequences: the rows of eight ids
        _case("embed-step", op="embed", n=8, vocab=50_000, dim=1024),
        # a batch of prompts: word-like ids, long rows, one id in 64 bits each
        _case("embed-prompts", op="embed", n=16_384, vocab=128_000, dim=4096, wide=True),
        # a small model's gradient, all in 32 bits
        _case("embed-grad-small", op="embed_grad", n=500, vocab=10_000, dim=256, type="f32", out="f32"),
        # a training batch's gradient: 16-bit rows summed into a 32-bit gradient; hot ids fill long runs
        _case("embed-grad-batch", op="embed_grad", n=65_536, vocab=50_000, dim=2048, type="bf16", out="f32"),
        # an SGD step on a large table of which a batch touches little (the zipf-1m workload's features)
        _case("embed-update", op="embed_update", n=8191, vocab=1_000_000, dim=320, type="bf16", out="f32", s=1.1),
        # a decoding step of four sequences under a grammar, with the alternatives that an API returns
        _case("logprobs-step", op="logprobs", n=4, vocab=128_000, k=20, masked=0.5),
        # scoring prompts, odd vocabulary, rows that start at any two bytes
        _case("logprobs-score", op="logprobs", n=2039, vocab=50_001, k=5),
        # the policy step of reinforcement learning: log probabilities, entropy and their gradient
        _case("logprobs-train", op="logprobs_train", n=4096, vocab=128_000),
        # a small student in 32 bits, eight teacher logits a row, no bucket for the rest
        _case("distill-small", op="distill", n=24, vocab=10_000, type="f32", k=8, grad=True),
        # the loss alone, on held-out rows, in half precision
        _case("distill-eval", op="distill", n=1024, vocab=32_000, type="f16", k=64, bucket=True, temperature=2.0),
        # an odd vocabulary, 32 bits, with gradient
        _case("distill-odd", op="distill", n=1501, vocab=50_001, type="f32", k=100, grad=True, bucket=True),
        # a training batch over a large vocabulary, with gradient
        _case("distill-batch", op="distill", n=4096, vocab=128_000, k=64, grad=True, bucket=True, temperature=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_update", "logprobs", "logprobs_train", "distill", "distill"])
    if op.startswith("embed"):
        dim = rng.choice([_log(rng, 32, 512), 40 * _log(rng, 1, 100)])
        vocab = _log(rng, 1000, 128_000) if op != "embed_update" else _log(rng, 10_000, 1_000_000)
        vocab = min(vocab, 100_000_000 // dim)
        n = min(_log(rng, 1, 65_536), 120_000_000 // dim)
        table = rng.choice(["f32", "bf16", "f16"])
        out = rng.choice([table, "f32"]) if op != "embed" else rng.choice([table, "bf16"])
        return _case(op=op, n=n, vocab=vocab, dim=dim, type=table, out=out, s=rng.choice([0.0, 1.0, 1.1]),
                     wide=rng.random() < 0.5)
    vocab = _log(rng, 2000, 128_000)
    n = min(_log(rng, 1, 8192), 400_000_000 // vocab)
    c = dict(op=op, n=n, vocab=vocab, type=rng.choice(["f32", "bf16", "bf16", "f16"]), wide=rng.random() < 0.5,
             temperature=rng.choice([1.0, 1.0, 0.7, 2.0]))
    if op == "logprobs":
        return _case(k=rng.choice([0, 1, 5, 20, 32]), masked=rng.choice([0.0, 0.0, 0.5, 0.9]), **c)
    if op == "logprobs_train":
        return _case(**c)
    return _case(k=_log(rng, 4, 200), grad=rng.random() < 0.7, bucket=rng.random() < 0.6, **c)


# ------------------------------------------------------------------ inputs
def _ids(n, vocab, s, g):
    """n ids, Zipf of exponent s over a random permutation of the vocabulary (s = 0: uniform)."""
    weight = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -s
    cum = torch.cumsum(weight, 0)
    u = torch.rand(n, device="cuda", dtype=torch.float64, generator=g) * cum[-1]
    rank = torch.searchsorted(cum, u).clamp_(max=vocab - 1)
    return torch.randperm(vocab, device="cuda", generator=g)[rank]


def _logits(n, vocab, g):
    """32-bit logits: noise, and four raised tokens in each row, the first of them most (returned with their places)."""
    z = torch.randn(n, vocab, device="cuda", generator=g) * 2.0
    at = torch.randint(0, vocab, (n, 4), device="cuda", generator=g)
    z.scatter_add_(1, at, torch.rand(n, 4, device="cuda", generator=g) * torch.tensor([12.0, 9.0, 7.0, 6.0], device="cuda"))
    return z, at


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, n, vocab, dim = case["op"], case["n"], case["vocab"], case["dim"]
    a, b = TYPES[case["type"]], TYPES[case["out"]]
    whole = torch.int64 if case["wide"] else torch.int32
    st = {"case": case}
    if op.startswith("embed"):
        st["ids"] = _ids(n, vocab, case["s"], g).to(whole)
        if op == "embed":
            st["table"] = (torch.randn(vocab, dim, device="cuda", generator=g) * 0.02).to(a)
            st["out"] = torch.empty(n, dim, device="cuda", dtype=b)
            st["scale"] = math.sqrt(dim)
        else:
            st["dout"] = (torch.randn(n, dim, device="cuda", generator=g) * 0.01).to(a)
            if op == "embed_update":
                st["table"] = (torch.randn(vocab, dim, device="cuda", generator=g) * 0.02).to(b)
                st["scale"] = -0.1 * math.sqrt(dim)
            else:
                st["table"] = torch.empty(vocab, dim, device="cuda", dtype=b)
                st["scale"] = math.sqrt(dim)
    else:
        z, at = _logits(n, vocab, g)
        st["scale"] = 1.0 / case["temperature"]
        if op == "distill":
            # early in training: the teacher is surer of the raised tokens, and differs by a noise of its own
            teacher = z + 1.5 * torch.randn(n, vocab, device="cuda", generator=g)
            teacher.scatter_add_(1, at[:, :1], torch.full((n, 1), 4.0, device="cuda"))
            st["top_logits"], top = torch.topk(teacher, case["k"], dim=1)
            st["top_ids"] = top.to(whole)
            st["teacher_lse"] = torch.logsumexp(teacher * st["scale"], 1) if case["bucket"] else None
            del teacher
            # rows of the padding at the end of sequences: the teacher has nothing to say, and their weight is zero
            pad = torch.rand(n, device="cuda", generator=g) < 0.03
            st["top_ids"][pad] = -1
            st["weight"] = torch.where(pad, 0.0, 1.0 / n) if case["grad"] else None
            st["loss"] = torch.empty(n, device="cuda")
        else:
            st["ids"] = at[:, 0].to(whole)
            if case["masked"]:
                drop = torch.rand(n, vocab, device="cuda", generator=g) < case["masked"]
                drop.scatter_(1, at, False)
                z.masked_fill_(drop, -math.inf)
                del drop
            st["logp"], st["lse"], st["entropy"] = (torch.empty(n, device="cuda") for _ in range(3))
            if case["k"]:
                st["top_logp"] = torch.empty(n, case["k"], device="cuda")
                st["top_ids"] = torch.empty(n, case["k"], device="cuda", dtype=torch.int32)
            if op == "logprobs_train":
                st["dlogp"] = torch.randn(n, device="cuda", generator=g) / n
                st["dentropy"] = torch.full((n,), 0.01 / n, device="cuda")
        st["logits"] = z.to(a)
        del z
        if op == "logprobs_train" or case["grad"]:
            st["dlogits"] = torch.empty_like(st["logits"])
    if own:
        import paper_1508_00703_gb300 as pdb
        st["tokens"] = pdb.pdb_tokens_create(n, max(dim, 1))
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_1508_00703_gb300 as pdb
    c, tok = st["case"], st["tokens"]
    op = c["op"]
    if op == "embed":
        pdb.pdb_embed(tok, st["table"], st["ids"], st["out"], scale=st["scale"])
        return st["out"]
    if op in ("embed_grad", "embed_update"):
        pdb.pdb_embed_grad(tok, st["ids"], st["dout"], st["table"], scale=st["scale"], accumulate=op == "embed_update")
        return st["table"]
    if op == "distill":
        pdb.pdb_distill(tok, st["logits"], st["top_ids"], st["top_logits"], st["loss"], teacher_lse=st["teacher_lse"],
                        weight=st["weight"], dlogits=st.get("dlogits"), temperature=c["temperature"])
        return {"loss": st["loss"], "dlogits": st.get("dlogits")}
    pdb.pdb_logprobs(tok, st["logits"], st["ids"], st["logp"], lse=st["lse"], entropy=st["entropy"],
                     top_logp=st.get("top_logp"), top_ids=st.get("top_ids"), scale=st["scale"])
    got = {m: st.get(m) for m in ("logp", "lse", "entropy", "top_logp", "top_ids")}
    if op == "logprobs_train":
        pdb.pdb_logprobs_grad(tok, st["logits"], st["ids"], st["lse"], st["entropy"], st["dlogp"], st["dentropy"],
                              st["dlogits"], scale=st["scale"])
        got["dlogits"] = st["dlogits"]
    return got


def _run_plain(st):
    c = st["case"]
    op, scale = c["op"], st["scale"]
    if op == "embed":
        return (st["table"][st["ids"].long()].float() * scale).to(st["out"].dtype)
    if op == "embed_grad":
        d = torch.zeros(c["vocab"], c["dim"], device="cuda")
        d.index_add_(0, st["ids"].long(), st["dout"].float() * scale)
        return d.to(st["table"].dtype)
    if op == "embed_update":
        # the touched rows alone: their sums, by the place of an id among the batch's distinct ones
        seen, place = torch.unique(st["ids"].long(), return_inverse=True)
        d = torch.zeros(seen.numel(), c["dim"], device="cuda")
        d.index_add_(0, place, st["dout"].float() * scale)
        st["table"][seen] = (st["table"][seen].float() + d).to(st["table"].dtype)
        return st["table"]
    z = st["logits"].float() * scale
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    if op == "distill":
        return _plain_distill(st, z - top, torch.log(total), e / total)
    p = e / total
    got = {"logp": z.gather(1, st["ids"].long()[:, None]).squeeze(1) - lse, "lse": lse,
           "entropy": lse - torch.where(p > 0, p * z, 0.0).sum(1)}
    if c["k"]:
        bits = (st["logits"].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF)
        key = order * 2 ** 32 + (c["vocab"] - 1 - torch.arange(c["vocab"], device="cuda"))
        best = c["vocab"] - 1 - torch.topk(key, c["k"], dim=1).values % 2 ** 32
        got["top_logp"] = z.gather(1, best) - lse[:, None]
        got["top_ids"] = best.int()
    if op == "logprobs_train":
        dlogp, dentropy = st["dlogp"][:, None], st["dentropy"][:, None]
        d = -p * (dlogp + dentropy * (z - lse[:, None] + got["entropy"][:, None]))
        d.scatter_add_(1, st["ids"].long()[:, None], dlogp)
        got["dlogits"] = (d * scale).to(st["logits"].dtype)
    return {m: got.get(m) for m in ("logp", "lse", "entropy", "top_logp", "top_ids", "dlogits")}


def _plain_distill(st, z, logtotal, p):
    # z less its row's maximum, the logarithm of the row's sum of exponentials, the probabilities
    T = st["case"]["temperature"]
    there = st["top_ids"] >= 0
    at = st["top_ids"].long().clamp(min=0)
    t = torch.where(there, st["top_logits"] / T, -math.inf)
    some = there.any(1)
    if st["teacher_lse"] is not None:
        logq = t - st["teacher_lse"][:, None]
        q = torch.exp(logq)
    else:
        peak = torch.where(some, t.amax(1), 0.0)[:, None]
        q = torch.exp(t - peak)
        all_q = torch.where(some, q.sum(1), 1.0)[:, None]
        logq, q = t - peak - torch.log(all_q), q / all_q
    loss = torch.where(q > 0, q * (logq - (z.gather(1, at) - logtotal)), 0.0).sum(1)
    factor = torch.ones_like(loss)
    if st["teacher_lse"] is not None:
        # the bucket: what the teacher's slots leave, against the student's probability outside of them
        inside = torch.zeros(z.shape, device="cuda", dtype=torch.bool).scatter_(1, at, there)
        rest_q = 1.0 - q.sum(1)
        rest_p = torch.where(inside, 0.0, p).sum(1)
        loss = loss + torch.where(rest_q > 1e-6, rest_q * torch.log(rest_q / rest_p), 0.0)
        factor = torch.where(rest_q > 1e-6, 1.0 - rest_q / rest_p, 1.0)
    got = {"loss": torch.where(some, T * T * loss, 0.0)}
    if st["weight"] is not None:
        d = p * factor[:, None]
        if st["teacher_lse"] is not None:
            d = torch.where(inside, p, d)
        d.scatter_add_(1, at, -q)
        got["dlogits"] = (torch.where(some[:, None], d, 0.0) * (st["weight"] * T)[:, None]).to(st["logits"].dtype)
    return {m: got.get(m) for m in ("loss", "dlogits")}


# ------------------------------------------------------------------ work and exact results
def work(case):
    op, n, vocab, dim, k = (case[m] for m in ("op", "n", "vocab", "dim", "k"))
    a, b = (4 if case[m] == "f32" else 2 for m in ("type", "out"))
    ids = n * (8 if case["wide"] else 4)
    if op.startswith("embed"):
        # distinct ids expected of n draws from the Zipf distribution
        rank = torch.arange(1, vocab + 1, dtype=torch.float64) ** -case["s"]
        seen = float((1.0 - torch.exp(n * torch.log1p(-(rank / rank.sum()).clamp(max=1 - 1e-12)))).sum())
        if op == "embed":
            return {"bytes": ids + seen * dim * a + n * dim * b, "flops": n * dim}
        written = vocab * dim * b if op == "embed_grad" else 2 * seen * dim * b
        return {"bytes": ids + n * dim * a + written, "flops": 2 * n * dim}
    cells = n * vocab
    if op == "distill":
        rows = n * k * (4 + (8 if case["wide"] else 4)) + n * 4 * (1 + case["grad"] + case["bucket"])
        return {"bytes": cells * a * (2 if case["grad"] else 1) + rows, "flops": cells * (8 if case["grad"] else 4)}
    if op == "logprobs":
        return {"bytes": cells * a + ids + n * (12 + 8 * k), "flops": cells * 6}
    return {"bytes": cells * a * 2 + ids + n * 20, "flops": cells * 12}


def _rows_of(n, vocab):
    """Row ranges of about 2^26 cells, so that 64-bit copies stay small."""
    step = max(1, 2 ** 26 // vocab)
    return [(i, min(n, i + step)) for i in range(0, n, step)]


def exact(case, seed):
    st = prepare(case, seed)
    op, n, vocab, dim = (case[m] for m in ("op", "n", "vocab", "dim"))
    if op.startswith("embed"):
        ids = st["ids"].long()
        if op == "embed":
            return st["table"].index_select(0, ids).double().mul_(st["scale"])
        base = st["table"].double() if op == "embed_update" else torch.zeros(vocab, dim, device="cuda", dtype=torch.float64)
        return base.index_put_((ids,), st["dout"].double() * st["scale"], accumulate=True)
    parts = []
    for r0, r1 in _rows_of(n, vocab):
        z = st["logits"][r0:r1].double() * st["scale"]
        z.requires_grad_(True)
        logp = torch.log_softmax(z, 1)
        if op == "distill":
            parts.append(_exact_distill(st, r0, r1, z, logp))
            continue
        at = st["ids"][r0:r1].long()[:, None]
        given = logp.gather(1, at).squeeze(1)
        held = logp.masked_fill(torch.isinf(logp), 0.0)
        entropy = -(logp.exp() * held).sum(1)
        out = {"logp": given, "lse": torch.logsumexp(z, 1), "entropy": entropy}
        if case["k"]:
            best = torch.sort(st["logits"][r0:r1].float(), dim=1, descending=True, stable=True).indices[:, :case["k"]]
            out["top_logp"] = logp.gather(1, best)
            out["top_ids"] = best.int()
        if op == "logprobs_train":
            total = (given * st["dlogp"][r0:r1]).sum() + (entropy * st["dentropy"][r0:r1]).sum()
            out["dlogits"] = torch.autograd.grad(total, z)[0] * st["scale"]
        parts.append({m: v.detach() for m, v in out.items()})
    names = ("loss", "dlogits") if op == "distill" else ("logp", "lse", "entropy", "top_logp", "top_ids", "dlogits")
    return {m: torch.cat([x[m] for x in parts]) if m in parts[0] else None for m in names}


def _exact_distill(st, r0, r1, z, logp):
    T = st["case"]["temperature"]
    ids = st["top_ids"][r0:r1].long()
    # the teacher's distribution laid out over the whole vocabulary, one column more taking the empty slots
    vocab = z.shape[1]
    t = st["top_logits"][r0:r1].double() / T
    put = torch.where(ids < 0, vocab, ids)
    full = torch.full((r1 - r0, vocab + 1), -math.inf, device="cuda", dtype=torch.float64).scatter_(1, put, t)[:, :vocab]
    live = (ids >= 0).any(1)
    if st["teacher_lse"] is None:
        logq = full - torch.where(live, torch.logsumexp(full, 1), 0.0)[:, None]
    else:
        logq = full - st["teacher_lse"][r0:r1].double()[:, None]
    q = logq.exp()
    inside = q > 0
    kl = (q * (logq.masked_fill(~inside, 0.0) - logp)).sum(1)
    if st["teacher_lse"] is not None:
        rest = 1.0 - q.sum(1)
        use = (rest > 1e-6) & live
        outside = torch.logsumexp(torch.where(inside, -math.inf, logp), 1)
        safe = torch.where(use, rest, 1.0)
        kl = kl + torch.where(use, safe * (torch.log(safe) - outside), 0.0)
    loss = torch.where(live, T * T * kl, 0.0)
    out = {"loss": loss.detach()}
    if st["weight"] is not None:
        out["dlogits"] = torch.autograd.grad((loss * st["weight"][r0:r1].double()).sum(), z)[0] / T
    return out
