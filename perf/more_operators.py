"""Drafted tokens verified, tokens sent to experts and back, gradients clipped: as a program that trains a token model with
experts and then drafts with it calls these operators, and their plain forms.

  op          verify      accepted drafts and the token drawn after them, from rows of logits and given random numbers,
                          and the log probabilities of these tokens
              route       places of the tokens' slots by expert, and the tokens' rows put there
              join        the experts' rows weighted and summed for each token
              join_train  the gradients of both: rows and weights of the join, the tokens' rows of the way in
              clip        norm over many gradients, and each of them, clipped to it, added to a weight or written

  Logits are a broad noise with a few raised tokens per row; the draft's logits are the target's with a noise of their own, and
  drafted tokens are drawn from them, so about four of five are accepted (with the draft looked up in the text, seven of ten are
  the target's favourite).  Experts are chosen by scores with a bias per expert; a few tokens are padding.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name=None, **kw):
    c = dict(op="verify", n=1, type="bf16", out="bf16", wide=False,
             vocab=0, drafts=0, lookup=False, ragged=False, masked=0.0, temperature=1.0,
             dim=0, k=0, experts=0, capacity=0,
             model="", layers=0, accumulate=False, clip=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence under a grammar, four drafts: the call whose latency a reader waits for
        _case("verify-step", op="verify", n=1, drafts=4, vocab=128_000, masked=0.5),
        # drafts looked up in the text (no draft model), eight for each of sixteen sequences, as many as matched
        _case("verify-lookup", op="verify", n=16, drafts=8, vocab=32_000, type="f16", lookup=True, ragged=True),
        # an odd vocabulary in 32 bits, a lower temperature, sequences that end early
        _case("verify-odd", op="verify", n=37, drafts=3, vocab=50_001, type="f32", temperature=0.7, ragged=True),
        # a server's batch
        _case("verify-batch", op="verify", n=256, drafts=5, vocab=128_000),
        # one decoding step of eight sequences
        _case("route-step", op="route", n=8, dim=1024, k=2, experts=16),
        # a training batch, many experts
        _case("route-batch", op="route", n=16_384, dim=2048, k=8, experts=64),
        # experts of a fixed capacity (one batched product over them), odd rows in 32 bits
        _case("route-capacity", op="route", n=4099, dim=1001, k=2, experts=32, capacity=300, type="f32", out="f32", wide=True),
        # the way back of a few tokens
        _case("join-step", op="join", n=65, dim=1024, k=4, experts=16, out="f32"),
        # backward of a training batch
        _case("join-train", op="join_train", n=8192, dim=4096, k=4, experts=64),
        # the token model of the examples: a table, an output matrix and a bias, all in 32 bits
        _case("clip-small", op="clip", model="tokens", dim=64, vocab=2000, type="f32", out="f32", accumulate=True),
        # a table's gradient in which a batch has touched little, and the output matrix, clipped into 16 bits for the exchange
        _case("clip-table", op="clip", model="tokens", dim=1025, vocab=50_001, type="f32", out="bf16"),
        # a model of many layers, gradients in 16 bits, the SGD step on weights in 32
        _case("clip-layers", op="clip", model="layers", dim=2048, vocab=32_000, layers=7, type="bf16", out="f32",
              accumulate=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["verify", "verify", "route", "join", "join_train", "clip"])
    if op == "verify":
        vocab, drafts = _log(rng, 1000, 128_000), rng.choice([0, 1, 2, 3, 4, 5, 8])
        n = min(_log(rng, 1, 512), 150_000_000 // (vocab * (drafts + 1)))
        return _case(op=op, n=max(n, 1), drafts=drafts, vocab=vocab, type=rng.choice(["f32", "bf16", "bf16", "f16"]),
                     lookup=rng.random() < 0.3, ragged=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.5, 0.9]),
                     temperature=rng.choice([1.0, 1.0, 0.7, 1.5]), wide=rng.random() < 0.5)
    if op == "clip":
        model = rng.choice(["tokens", "layers"])
        dim = _log(rng, 33, 2048) if model == "tokens" else 8 * _log(rng, 4, 200)
        vocab = min(_log(rng, 500, 100_000), 100_000_000 // dim)
        a = rng.choice(["f32", "bf16", "f16"])
        return _case(op=op, model=model, dim=dim, vocab=vocab, layers=_log(rng, 1, 7) if model == "layers" else 0, type=a,
                     out=rng.choice([a, "f32"]), accumulate=rng.random() < 0.6, clip=rng.choice([1.0, 1.0, 1e6]))
    k, experts = rng.choice([1, 2, 4, 6, 8]), rng.choice([8, 16, 60, 64, 128, 256])
    dim = rng.choice([_log(rng, 32, 512), 40 * _log(rng, 1, 100)])
    n = min(_log(rng, 1, 32_768), 200_000_000 // (dim * k))
    a = rng.choice(["f32", "bf16", "bf16", "f16"])
    capacity = rng.choice([0, 0, max(1, math.ceil(1.25 * n * k / experts))])
    return _case(op=op, n=n, dim=dim, k=k, experts=experts, capacity=capacity, type=a, out=rng.choice([a, a, "f32"]),
                 wide=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _shapes(case):
    """The gradients of a model, by shape, and whether a batch touches few rows of it."""
    dim, vocab = case["dim"], case["vocab"]
    ends = [((vocab, dim), True), ((vocab, dim), False), ((vocab,), False)]
    layer = [((dim,), False), ((3 * dim, dim), False), ((dim, dim), False), ((dim,), False), ((4 * dim, dim), False),
             ((4 * dim,), False), ((dim, 4 * dim), False), ((dim,), False)]
    return ends + layer * case["layers"]


def _places(ids, experts, capacity):
    """place (n, k), source (rows), ends (experts) of the slots' experts, by a stable sort."""
    n, k = ids.shape
    e = ids.long().reshape(-1)
    e = torch.where(e >= 0, e, experts)
    rows = experts * capacity if capacity else n * k
    count = (e[:, None] == torch.arange(experts, device=e.device)).sum(0)
    before = torch.cat([count.new_zeros(1), count.cumsum(0)])             # slots of lower experts
    order = torch.sort(e, stable=True).indices
    rank = torch.empty_like(e)
    rank[order] = torch.arange(n * k, device=e.device) - before[e[order]]
    if capacity:
        first = torch.arange(experts + 1, device=e.device) * capacity
        ends = first[:experts] + count.clamp(max=capacity)
        kept = (e < experts) & (rank < capacity)
    else:
        first, ends, kept = before, before[1:], e < experts
    place = torch.where(kept, first[e] + rank, -1)
    source = torch.full((rows,), -1, device=e.device, dtype=torch.int32)
    source[place[kept]] = kept.nonzero().squeeze(1).int()
    return place.view(n, k).int(), source, ends.int()


def _prepare_verify(st, g):
    c = st["case"]
    n, D, vocab, dtype = c["n"], c["drafts"], c["vocab"], TYPES[c["type"]]
    st["scale"] = 1.0 / c["temperature"]
    z = torch.randn(n * (D + 1), vocab, device="cuda", generator=g) * 2.0
    at = torch.randint(0, vocab, (n * (D + 1), 4), device="cuda", generator=g)
    z.scatter_add_(1, at, torch.rand(at.shape, device="cuda", generator=g) * torch.tensor([12.0, 9.0, 7.0, 6.0], device="cuda"))
    if c["masked"]:
        drop = torch.rand(z.shape, device="cuda", generator=g) < c["masked"]
        drop.scatter_(1, at, False)
        z.masked_fill_(drop, -math.inf)
        del drop
    st["target"] = z.to(dtype)
    z = z.view(n, D + 1, vocab)[:, :D].reshape(n * D, vocab)
    st["draft"] = None
    if c["lookup"]:
        best = z.argmax(1) if D else torch.zeros(0, device="cuda", dtype=torch.int64)
        other = torch.randint(0, vocab, (n * D,), device="cuda", generator=g)
        ids = torch.where(torch.rand(n * D, device="cuda", generator=g) < 0.7, best, other)
    else:
        st["draft"] = (z + 0.5 * torch.randn(z.shape, device="cuda", generator=g)).to(dtype)
        q = torch.softmax(st["draft"].float() * st["scale"], 1)
        ids = torch.multinomial(q, 1, generator=g).squeeze(1) if D else torch.zeros(0, device="cuda", dtype=torch.int64)
        del q
    ids = ids.view(n, D)
    if c["ragged"] and D:
        length = torch.randint(0, D + 1, (n, 1), device="cuda", generator=g)
        ids = torch.where(torch.arange(D, device="cuda") < length, ids, -1)
    st["ids"] = ids.to(torch.int64 if c["wide"] else torch.int32)
    st["accept"] = torch.rand(n, D, device="cuda", generator=g)
    st["pick"] = torch.rand(n, device="cuda", generator=g)
    st["tokens"] = torch.empty(n, D + 1, device="cuda", dtype=torch.int32)
    st["accepted"] = torch.empty(n, device="cuda", dtype=torch.int32)
    st["logp"] = torch.empty(n, D + 1, device="cuda")


def _prepare_experts(st, g):
    c = st["case"]
    n, k, dim, experts = c["n"], c["k"], c["dim"], c["experts"]
    a, b = TYPES[c["type"]], TYPES[c["out"]]
    scores = torch.randn(n, experts, device="cuda", generator=g) + 0.5 * torch.randn(experts, device="cuda", generator=g)
    top, ids = torch.topk(scores, k, dim=1)
    ids[torch.rand(n, device="cuda", generator=g) < 0.03] = -1            # padding
    st["ids"] = ids.to(torch.int64 if c["wide"] else torch.int32)
    rows = experts * c["capacity"] if c["capacity"] else n * k

    def values(m, dtype):
        return torch.randn(m, dim, device="cuda", generator=g).to(dtype)
    if c["op"] == "route":
        st["x"] = values(n, a)
        st["place"] = torch.empty(n, k, device="cuda", dtype=torch.int32)
        st["source"] = torch.empty(rows, device="cuda", dtype=torch.int32)
        st["ends"] = torch.empty(experts, device="cuda", dtype=torch.int32)
        st["rows"] = torch.empty(rows, dim, device="cuda", dtype=b)
        return
    st["place"], st["source"], _ = _places(st["ids"], experts, c["capacity"])
    st["weight"] = torch.softmax(top, 1)
    st["rows"] = values(rows, a)
    if c["op"] == "join":
        st["y"] = torch.empty(n, dim, device="cuda", dtype=b)
    else:
        st["dy"], st["din"] = values(n, b), values(rows, a)
        st["drows"], st["dweight"] = torch.empty_like(st["rows"]), torch.empty(n, k, device="cuda")
        st["dx"] = torch.empty(n, dim, device="cuda", dtype=b)


def _prepare_clip(st, g):
    c = st["case"]
    a, b = TYPES[c["type"]], TYPES[c["out"]]
    st["grads"], st["outs"] = [], []
    for i, (shape, sparse) in enumerate(_shapes(c)):
        d = torch.randn(shape, device="cuda", generator=g) * (0.002 * (1 + i % 5))
        if sparse:
            d *= (torch.rand(shape[0], 1, device="cuda", generator=g) < 0.1).float()
        st["grads"].append(d.to(a))
        del d
        st["outs"].append((torch.randn(shape, device="cuda", generator=g) * 0.02).to(b) if c["accumulate"]
                          else torch.empty(shape, device="cuda", dtype=b))
    st["norm"] = torch.empty(1, device="cuda")
    st["scale"] = -0.1 if c["accumulate"] else 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = {"case": case}
    op = case["op"]
    if op == "verify":
        _prepare_verify(st, g)
    elif op == "clip":
        _prepare_clip(st, g)
    else:
        _prepare_experts(st, g)
    if own:
        import paper_1508_00703_gb300 as pdb
        if op == "clip":
            st["plan"] = pdb.pdb_clip_plan_build(st["grads"], st["outs"])
        else:
            st["tok"] = pdb.pdb_tokens_create(case["n"] * max(case["k"], 1), 0)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_1508_00703_gb300 as pdb
    c = st["case"]
    op = c["op"]
    if op == "clip":
        pdb.pdb_clip(st["plan"], c["clip"], st["norm"], scale=st["scale"], accumulate=c["accumulate"])
        return {"norm": st["norm"], "outs": st["outs"]}
    tok = st["tok"]
    if op == "verify":
        pdb.pdb_verify(tok, st["target"], st["ids"], st["accept"], st["pick"], st["tokens"], st["accepted"], draft=st["draft"],
                       scale=st["scale"], draft_scale=st["scale"], logp=st["logp"])
        return {m: st[m] for m in ("tokens", "accepted", "logp")}
    if op == "route":
        pdb.pdb_route(tok, st["ids"], c["experts"], st["place"], st["source"], st["ends"], capacity=c["capacity"])
        pdb.pdb_route_rows(tok, st["x"], st["place"], st["source"], st["rows"])
        return {m: st[m] for m in ("place", "source", "ends", "rows")}
    if op == "join":
        pdb.pdb_route_join(tok, st["rows"], st["place"], st["y"], weight=st["weight"])
        return st["y"]
    pdb.pdb_route_join_grad(tok, st["rows"], st["place"], st["source"], st["dy"], st["drows"], weight=st["weight"],
                            dweight=st["dweight"])
    pdb.pdb_route_join(tok, st["din"], st["place"], st["dx"])
    return {m: st[m] for m in ("drows", "dweight", "dx")}


def _run_plain(st):
    c = st["case"]
    op = c["op"]
    if op == "verify":
        return _plain_verify(st)
    if op == "clip":
        return _plain_clip(st)
    if op == "route":
        place, source, ends = _places(st["ids"], c["experts"], c["capacity"])
        rows = st["x"].float()[(source // c["k"]).long().clamp(min=0)]
        rows = torch.where(source[:, None] >= 0, rows, 0.0).to(st["rows"].dtype)
        return {"place": place, "source": source, "ends": ends, "rows": rows}
    there, at = st["place"] >= 0, st["place"].long().clamp(min=0)
    w = torch.where(there, st["weight"], 0.0)
    if op == "join":
        y = torch.zeros(st["y"].shape, device="cuda")
        for j in range(c["k"]):
            y += w[:, j:j + 1] * st["rows"][at[:, j]].float()
        return y.to(st["y"].dtype)
    dy = st["dy"].float()
    dweight, dx = torch.zeros_like(w), torch.zeros_like(dy)
    for j in range(c["k"]):
        dweight[:, j] = torch.where(there[:, j], (dy * st["rows"][at[:, j]].float()).sum(1), 0.0)
        dx += torch.where(there[:, j:j + 1], st["din"][at[:, j]].float(), 0.0)
    source = st["source"].long()
    slot = source.clamp(min=0)
    drows = torch.where(source[:, None] >= 0, w.view(-1)[slot][:, None] * dy[slot // c["k"]], 0.0)
    return {"drows": drows.to(st["drows"].dtype), "dweight": dweight, "dx": dx.to(st["dx"].dtype)}


def _plain_softmax(z, scale):
    # in 64 bits: whether a number lies below a probability or a sum of them decides which token comes out
    z = z.double() * scale
    e = torch.exp(z - z.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_verify(st):
    c = st["case"]
    n, D, vocab = c["n"], c["drafts"], c["vocab"]
    ids = st["ids"].long()
    p = _plain_softmax(st["target"], st["scale"]).view(n, D + 1, vocab)
    there = (ids >= 0).cumprod(1)
    length = there.sum(1)
    at = ids.clamp(min=0)[:, :, None]
    p_at = p[:, :D].gather(2, at).squeeze(2)
    if st["draft"] is not None:
        q = _plain_softmax(st["draft"], st["scale"]).view(n, D, vocab)
        q_at = q.gather(2, at).squeeze(2)
    else:
        q, q_at = None, torch.ones_like(p_at)
    good = (st["accept"].double() * q_at < p_at) & (there > 0)
    a = good.long().cumprod(1).sum(1)
    row = torch.arange(n, device="cuda")
    r = p[row, a]
    refused = a < length
    if D:
        last = a.clamp(max=D - 1)
        less = torch.zeros_like(r).scatter_(1, ids.clamp(min=0)[row, last][:, None], 1.0) if q is None else q[row, last]
        r = torch.where(refused[:, None], (r - less).clamp(min=0.0), r)
    total = r.cumsum(1)
    drawn = (total <= st["pick"].double()[:, None] * total[:, -1:]).sum(1).clamp(max=vocab - 1)
    j = torch.arange(D + 1, device="cuda")
    kept = torch.cat([ids, torch.full((n, 1), -1, device="cuda", dtype=torch.int64)], 1)
    tokens = torch.where(j < a[:, None], kept, torch.where(j == a[:, None], drawn[:, None], -1))
    logp = torch.where(tokens >= 0, torch.log(p.gather(2, tokens.clamp(min=0)[:, :, None]).squeeze(2)), 0.0)
    return {"tokens": tokens.int(), "accepted": a.int(), "logp": logp.float()}


def _plain_clip(st):
    c = st["case"]
    total = torch.zeros(1, device="cuda", dtype=torch.float64)
    for d in st["grads"]:
        total += d.float().square().sum()
    norm = total.sqrt().float()
    factor = torch.where(norm > c["clip"], c["clip"] / norm, 1.0) * st["scale"]
    for d, o in zip(st["grads"], st["outs"]):
        v = d.float() * factor
        o.copy_(o.float() + v if c["accumulate"] else v)
    return {"norm": norm, "outs": st["outs"]}


# ------------------------------------------------------------------ work and exact results
def work(case):
    op, n, vocab, dim, k = (case[m] for m in ("op", "n", "vocab", "dim", "k"))
    a, b = (4 if case[m] == "f32" else 2 for m in ("type", "out"))
    if op == "verify":
        # positions up to the first refusal, four of five drafts accepted; sequences end early where they are ragged
        D, good = case["drafts"], 0.7 if case["lookup"] else 0.8
        lengths = range(D + 1) if case["ragged"] else [D]
        targets = sum(sum(good ** d for d in range(L + 1)) for L in lengths) / len(lengths)
        drafts = 0.0 if case["lookup"] else sum(sum(good ** d for d in range(L)) for L in lengths) / len(lengths)
        cells = n * (targets + drafts) * vocab
        return {"bytes": cells * a + n * (D + 1) * 16, "flops": cells * 4}
    if op == "clip":
        cells = sum(math.prod(shape) for shape, _ in _shapes(case))
        return {"bytes": cells * (a + b * (2 if case["accumulate"] else 1)), "flops": cells * 4}
    rows = case["experts"] * case["capacity"] if case["capacity"] else n * k
    filled = min(rows, n * k)
    if op == "route":
        plan = n * k * ((8 if case["wide"] else 4) + 4) + rows * 4 + case["experts"] * 4
        return {"bytes": plan + n * dim * a + rows * dim * b, "flops": n * k}
    if op == "join":
        return {"bytes": n * k * 8 + filled * dim * a + n * dim * b, "flops": 2 * n * k * dim}
    return {"bytes": n * k * 12 + rows * 4 + (2 * filled + rows) * dim * a + 2 * n * dim * b, "flops": 4 * n * k * dim}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(st)
    if case["op"] == "clip":
        flat = [d.double() for d in st["grads"]]
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(d) for d in flat]))
        factor = st["scale"] * min(1.0, case["clip"] / float(norm))
        outs = [d.mul_(factor).add_(o.double()) if case["accumulate"] else d.mul_(factor) for d, o in zip(flat, st["outs"])]
        return {"norm": norm.view(1), "outs": outs}
    return _exact_experts(st)


def _exact_verify(st):
    c = st["case"]
    n, D = c["n"], c["drafts"]
    ids, accept, pick = st["ids"].tolist(), st["accept"].tolist(), st["pick"].tolist()
    tokens, accepted = torch.full((n, D + 1), -1, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)
    logp = torch.zeros(n, D + 1, dtype=torch.float64)
    for s in range(n):
        a, rest = 0, None
        while True:
            l = torch.log_softmax(st["target"][s * (D + 1) + a].double() * st["scale"], 0)
            p = l.exp()
            if a == D or ids[s][a] < 0:
                rest = p
                break
            t = ids[s][a]
            if st["draft"] is None:
                q = torch.nn.functional.one_hot(torch.tensor(t, device="cuda"), c["vocab"]).double()
            else:
                q = torch.log_softmax(st["draft"][s * D + a].double() * st["scale"], 0).exp()
            if accept[s][a] * float(q[t]) >= float(p[t]):
                rest = torch.relu(p - q)
                break
            tokens[s, a], logp[s, a] = t, l[t]
            a += 1
        upto = torch.cumsum(rest, 0)
        drawn = torch.searchsorted(upto, upto[-1:] * pick[s], right=True)
        tokens[s, a] = min(int(drawn), c["vocab"] - 1)
        logp[s, a] = l[tokens[s, a]]
        accepted[s] = a
    return {"tokens": tokens.cuda(), "accepted": accepted.cuda(), "logp": logp.cuda()}


def _exact_experts(st):
    c = st["case"]
    n, k, experts, capacity = c["n"], c["k"], c["experts"], c["capacity"]
    if c["op"] == "route":
        flat = st["ids"].reshape(-1).cpu()
        rows = experts * capacity if capacity else n * k
        place, source = torch.full((n * k,), -1, dtype=torch.int32), torch.full((rows,), -1, dtype=torch.int32)
        ends = torch.zeros(experts, dtype=torch.int32)
        at = 0
        for e in range(experts):
            slots = (flat == e).nonzero().squeeze(1)
            if capacity:
                at, slots = e * capacity, slots[:capacity]
            here = torch.arange(at, at + slots.numel(), dtype=torch.int32)
            place[slots], source[here.long()] = here, slots.int()
            at += slots.numel()
            ends[e] = at
        x = torch.cat([st["x"].double(), torch.zeros(1, c["dim"], device="cuda", dtype=torch.float64)])
        token = torch.where(source < 0, n, source // k).long().cuda()
        return {"place": place.view(n, k).cuda(), "source": source.cuda(), "ends": ends.cuda(), "rows": x[token]}
    at = st["place"].long().reshape(-1)
    slot = (at >= 0).nonzero().squeeze(1)                  # slots that have a row, their rows, their tokens
    row, token = at[slot], slot // k
    w = st["weight"].double().reshape(-1)
    some = torch.arange(0, slot.numel(), max(1, 2 ** 26 // c["dim"])).tolist() + [slot.numel()]

    def summed(values, weights):
        y = torch.zeros(n, c["dim"], device="cuda", dtype=torch.float64)
        for i, j in zip(some, some[1:]):
            y.index_add_(0, token[i:j], values[row[i:j]].double() * weights[i:j, None])
        return y
    if c["op"] == "join":
        return summed(st["rows"], w[slot])
    drows = torch.zeros(st["rows"].shape, device="cuda", dtype=torch.float64)
    dweight = torch.zeros(n * k, device="cuda", dtype=torch.float64)
    for i, j in zip(some, some[1:]):
        dy = st["dy"][token[i:j]].double()
        drows[row[i:j]] = dy * w[slot[i:j], None]
        dweight[slot[i:j]] = torch.einsum("rd,rd->r", dy, st["rows"][row[i:j]].double())
    return {"drows": drows, "dweight": dweight.view(n, k), "dx": summed(st["din"], torch.ones_like(w[slot]))}
