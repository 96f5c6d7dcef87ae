"""Plain 64-bit forms of the token operators and how far fp32 arithmetic may be from them.

Every bound follows from the formula, with u = 2^-24 the unit roundoff of
fp32 and first-order error terms: an fp32 product or sum of exact operands is
off by u of its value; a sum of c terms in any order by at most (c - 1) u of
the sum of magnitudes (the kernels add at most cols / 128 + 64 terms one after
the other and join the partial sums pairwise or by thread, block and
cluster); exp and log are taken as good to 4 u (2 ulp); an argument d = (z - m) * scale
with two roundings moves exp(d) by 2 u |d|.  `slack` = 2 covers the second order
and the roundings of constants.  Outputs in 16 bits add half a unit of their type."""
import math

import torch

U = 2.0 ** -24
SLACK = 2.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place, relative, and the smallest step (subnormal) of a type
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def rounding(value, dtype):
    return HALF_ULP[dtype] * value.abs() + TINY[dtype]


def terms(cols):
    return cols / 128 + 64


def assert_near(got, want, tol, what):
    """|got - want| <= tol elementwise, infinities and NaN in the same places."""
    got, want, tol = got.double().cpu(), want.double().cpu(), tol.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN in other places"
    # a value that its bound takes past fp32's largest may come out infinite
    over = torch.isinf(got) & (want.abs() + tol > torch.finfo(torch.float32).max) & (got.sign() == want.sign())
    odd = (torch.isinf(want) | torch.isinf(got)) & ~over
    assert torch.equal(got[odd], want[odd]), what + ": infinities differ"
    ok = ~odd & ~over & ~torch.isnan(want)
    off = (got[ok] - want[ok]).abs() - tol.expand(want.shape)[ok]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: over the bound by {off.max():.3g}"


def embed_grad(ids, dout, vocab, scale, old=None, dtype=torch.float32, pad=-1):
    """(sum, bound): the ordered sums in 64 bits, on the CPU."""
    ids, d = ids.long().cpu(), dout.double().cpu()
    keep = (ids != pad) & (ids >= 0) & (ids < vocab)
    total = torch.zeros(vocab, d.shape[1], dtype=torch.float64)
    size = torch.zeros_like(total)
    count = torch.zeros(vocab, 1, dtype=torch.float64)
    total.index_add_(0, ids[keep], d[keep])
    size.index_add_(0, ids[keep], d[keep].abs())
    count.index_add_(0, ids[keep], torch.ones(int(keep.sum()), 1, dtype=torch.float64))
    s = float(torch.tensor(scale, dtype=torch.float32))
    want = s * total
    tol = SLACK * U * (count + 2) * abs(s) * size
    if old is not None:
        want = torch.where(count > 0, old.double().cpu() + want, old.double().cpu())
        tol = tol + torch.where(count > 0, U * want.abs(), 0.0)
    return want, tol + torch.where(count > 0, rounding(want, dtype), 0.0)


class Rows:
    """Softmax statistics of rows of logits in 64 bits, with bounds of the fp32 forms."""

    def __init__(self, logits, scale):
        s = float(torch.tensor(scale, dtype=torch.float32))
        self.raw = logits.double().cpu()
        self.z = self.raw * s
        self.cols = self.z.shape[1]
        self.none = (self.z == -math.inf).all(1)
        self.lse = torch.logsumexp(self.z, 1)
        bad = torch.isnan(self.z).any(1) | (self.z == math.inf).any(1)
        self.lse = torch.where(bad, math.nan, self.lse)
        m = torch.where(self.none, 0.0, self.z.amax(1))
        # by differences from the row's maximum: log p of logits near the type's lowest value would be lost beside lse
        self.logp = self.z - m[:, None]
        self.logp = self.logp - torch.where(self.none, 0.0, torch.logsumexp(self.logp, 1))[:, None]
        self.logp = torch.where(bad[:, None], math.nan, self.logp)
        self.p = self.logp.exp()
        held = torch.where(self.p > 0, self.logp, 0.0)
        self.held = torch.where(bad[:, None], math.nan, held)
        self.entropy = -(self.p * self.held).sum(1)
        d = torch.where(self.p > 0, self.z - m[:, None], 0.0)
        away = torch.nan_to_num(self.z - m[:, None], nan=0.0, posinf=0.0, neginf=0.0).abs()   # of any token, p = 0 too
        self.mean_d = (self.p * d.abs()).sum(1)
        mean_d2 = (self.p * d * d).sum(1)
        T = terms(self.cols)
        # relative error of the row's sum of exponentials, and with it of its logarithm
        self.rel_s = U * (2 * self.mean_d + 4 + T)
        log_s = (self.lse - m).abs()
        self.tol_lse = SLACK * (self.rel_s + U * (4 * log_s + 2 * m.abs() + self.lse.abs()))
        self.tol_logp = SLACK * ((self.rel_s + 5 * U * log_s)[:, None] + U * 4 * away)
        # entropy = log s - w / s, w = sum of e d
        self.tol_entropy = SLACK * (2 * self.rel_s + 5 * U * log_s + self.mean_d * (self.rel_s + 4 * U)
                                    + U * (2 * mean_d2 + (T + 6) * self.mean_d) + U * self.entropy.abs())
        self.tol_lse, self.tol_logp, self.tol_entropy = (torch.nan_to_num(t, nan=0.0, posinf=0.0) for t in
                                                        (self.tol_lse, self.tol_logp, self.tol_entropy))


def top(logits, k):
    """The k largest in each row: value descending (a NaN first), then the lower token."""
    z = logits.double().cpu() + 0.0
    z = torch.where(torch.isnan(z), math.inf, z)
    nan = torch.isnan(logits.double().cpu())
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    nan_first = torch.sort(nan.gather(1, order).int(), dim=1, descending=True, stable=True).indices
    return order.gather(1, nan_first)[:, :k]


def logprobs_grad(logits, ids, scale, lse, entropy, dlogp, dentropy, dtype, ignore=-100):
    """(gradient, bound) with lse and entropy taken as given (fp32 values)."""
    s = float(torch.tensor(scale, dtype=torch.float32))
    z = logits.double().cpu() * s
    n, cols = z.shape
    l = lse.double().cpu()[:, None]
    H = (entropy.double().cpu() if entropy is not None else torch.zeros(n, dtype=torch.float64))[:, None]
    g = (dlogp.double().cpu() if dlogp is not None else torch.zeros(n, dtype=torch.float64))[:, None].clone()
    h = (dentropy.double().cpu() if dentropy is not None else torch.zeros(n, dtype=torch.float64))[:, None]
    one = torch.zeros_like(z)
    if dlogp is not None:
        t = ids.long().cpu()
        there = (t != ignore) & (t >= 0) & (t < cols)
        g[~there] = 0.0
        one[torch.arange(n)[there], t[there]] = 1.0
    zero = ((g == 0) & (h == 0)) | (l == -math.inf)
    x = z - l
    p = x.exp()
    xh = torch.where(p == 0, 0.0, x)
    want = s * (g * (one - p) - h * p * (xh + torch.where(p == 0, 0.0, H)))
    rel_p = U * ((x - 0).abs() + z.abs() + 6)
    tol = SLACK * s * (g.abs() * (p * rel_p + 3 * U * (one + p))
                       + h.abs() * p * ((xh.abs() + H.abs()) * (rel_p + 6 * U) + U * (z.abs() + x.abs())))
    tol = torch.where(p == 0, SLACK * U * s * (g.abs() * one), tol)
    want = torch.where(zero, 0.0, want)
    tol = torch.where(zero, 0.0, tol + rounding(want, dtype) + abs(s) * (g.abs() + h.abs() * 128) * 2.0 ** -126)
    return want, torch.nan_to_num(tol, nan=0.0, posinf=0.0)


def distill(logits, top_ids, top_logits, teacher_lse, temperature, weight=None, dtype=torch.float32):
    """((loss, bound), (gradient, bound)) of the definition, slot by slot, in 64 bits."""
    T = float(torch.tensor(temperature, dtype=torch.float32))
    R = Rows(logits, 1.0 / T)
    n, cols = R.z.shape
    ids = top_ids.long().cpu().reshape(n, -1)
    K = ids.shape[1]
    used = (ids >= 0) & (ids < cols)
    t = torch.where(used, top_logits.double().cpu() / T, -math.inf)
    live = (t != -math.inf).any(1)
    at = torch.where(used, ids, 0)
    if teacher_lse is None:
        base = torch.where(live, torch.logsumexp(t, 1), 0.0)
    else:
        base = teacher_lse.double().cpu()
    lq = torch.where(used, t - base[:, None], -math.inf)
    q = lq.exp()
    x = R.logp.gather(1, at) if K else torch.zeros(n, 0, dtype=torch.float64)
    part = torch.where(q > 0, q * (torch.where(q > 0, lq, 0.0) - x), 0.0)
    part = torch.where(torch.isnan(q), math.nan, part)
    kl = part.sum(1)
    # q: two roundings of t / T, one of the difference, exp, and for the softmax the sum's and the quotient's
    tmax = torch.where(used & (t != -math.inf), t.abs(), 0.0)
    rel_q = U * (3 * tmax + 2 * torch.where(q > 0, lq.abs(), 0.0) + 2 * base.abs()[:, None] + 8)
    rel_q = rel_q + ((q * rel_q).sum(1, keepdim=True) + U * terms(K) if teacher_lse is None else 0.0)
    tol_x = R.tol_logp.gather(1, at) if K else torch.zeros(n, 0, dtype=torch.float64)
    lqx = torch.where(q > 0, (torch.where(q > 0, lq, 0.0) - x).abs(), 0.0)
    tol = (q * (rel_q * (1 + lqx) + tol_x + 4 * U * (lqx + torch.where(q > 0, lq.abs(), 0.0)))).sum(1)
    tol = tol + U * terms(K) * (q * lqx).sum(1)
    inside = torch.zeros(n, cols + 1, dtype=torch.bool).scatter_(1, torch.where(used, ids, cols), True)[:, :cols]
    factor = torch.ones(n, dtype=torch.float64)
    tol_f = torch.zeros(n, dtype=torch.float64)
    rest = torch.zeros(n, dtype=torch.float64)
    if teacher_lse is not None:
        rest = 1.0 - q.sum(1)
        rest = torch.where(rest <= 1e-6, 0.0, rest)
        tol_r = (q * rel_q).sum(1) + U * terms(K) * q.sum(1) + U
        logout = torch.logsumexp(torch.where(inside, -math.inf, R.logp), 1)
        on = rest > 0
        safe = torch.where(on, rest, 1.0)
        ratio = torch.where(on, torch.log(safe) - logout, 0.0)
        kl = kl + torch.where(on, safe * ratio, 0.0)
        tol_out = SLACK * (2 * R.rel_s + U * (8 + R.cols / 128 + 64)) + 8 * U * logout.abs()
        outside_d = torch.where(inside, 0.0, R.p * torch.where(R.p > 0, (R.logp - R.logp.amax(1, keepdim=True)).abs(), 0.0)).sum(1)
        tol_out = tol_out + SLACK * U * 4 * outside_d / logout.exp().clamp(min=1e-300)
        tol = tol + torch.where(on, tol_r * (1 + ratio.abs()) + rest * (tol_out + 8 * U * (safe.log().abs() + ratio.abs())), 0.0)
        finite = on & (logout > -math.inf)
        factor = torch.where(finite, 1.0 - safe / logout.exp(), 1.0)
        tol_f = torch.where(finite, safe / logout.exp() * (tol_r / safe + tol_out + 8 * U) + 2 * U, 0.0)
    loss = torch.where(live, torch.where(R.none, math.inf, T * T * kl), 0.0)
    tol_loss = SLACK * T * T * (tol + 4 * U * kl.abs()) + 1e-37
    tol_loss = torch.nan_to_num(tol_loss, nan=0.0, posinf=0.0)
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double().cpu()
    zero = (w == 0) | ~live | R.none
    dense = torch.where(inside, R.p, R.p * factor[:, None])
    qs = torch.zeros(n, cols + 1, dtype=torch.float64).scatter_add_(1, torch.where(used, ids, cols), q)[:, :cols]
    tol_q = torch.zeros(n, cols + 1, dtype=torch.float64).scatter_add_(1, torch.where(used, ids, cols), q * rel_q)[:, :cols]
    grad = (dense - qs) * (w * T)[:, None]
    rel_p = R.rel_s[:, None] + U * (2 * torch.where(R.p > 0, (R.logp - R.logp.amax(1, keepdim=True)).abs(), 0.0) + 8)
    tol_g = torch.where(inside, R.p * rel_p + tol_q + 4 * U * (R.p + qs),
                        R.p * (rel_p * factor.abs()[:, None] + tol_f[:, None] + 4 * U * factor.abs()[:, None]))
    tol_g = SLACK * tol_g * (w.abs() * T)[:, None]
    grad = torch.where(zero[:, None], 0.0, grad)
    tol_g = torch.where(zero[:, None], 0.0, tol_g + rounding(grad, dtype) + 2.0 ** -120 * (w.abs() * T)[:, None])
    return (loss, tol_loss), (grad, torch.nan_to_num(tol_g, nan=0.0, posinf=0.0))
