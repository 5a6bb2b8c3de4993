"""Log-probabilities of tokens, the policy loss and their gradients by their definitions in 64 bits, with bounds of what fp32 arithmetic
may be off by.

A row's sum of exponentials is off by SUM relative (chains of up to 64 terms a thread and at most 15 merges of two factors and three
roundings: (64 + 45) 2^-24 + 15 2^-22 < 1.2e-5), an exponential with exponent z by EXP |z| (2^-22 and four roundings of z).  So with
qo the mass of all other tokens, log q_token, which is a function of log sum_others - x_token, is off by qo times that and the roundings of
its parts, and four half steps of itself."""
import math

SUM, EXP, STEP = 1.2e-5, 2e-7, 2.0 ** -24
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
NEG = float("-inf")


class Rows:
    """l = log q_token, H and what they are made of, for [rows, V] logits; dl, dH: bounds."""

    def __init__(self, logits, tokens, tau):
        import torch
        x = logits.double() / tau
        V = x.shape[1]
        t = tokens.long()
        self.live = (t >= 0) & (t < V)
        self.t = t.clamp(0, V - 1)
        self.x, self.tau = x, tau
        self.xt = x.gather(1, self.t[:, None])[:, 0]
        others = x.scatter(1, self.t[:, None], NEG)
        m = others.max(-1).values
        self.empty = torch.isinf(m) & (m < 0) & torch.isinf(self.xt) & (self.xt < 0)
        safe = torch.where(torch.isinf(m) & (m < 0), 0.0, m)
        self.z = x - safe[:, None]                                     # exponents
        e = (others - safe[:, None]).exp()
        mass = e.sum(-1)
        # (against the largest of the others: differences of the type's lowest values are exact, their logarithms' sums are not)
        D = mass.log() - (self.xt - safe)
        D = torch.where(self.xt == math.inf, math.nan, D)
        D = torch.where(torch.isposinf(others).any(-1), math.nan, D)
        self.l = torch.where(self.empty, NEG, -torch.nn.functional.softplus(D, threshold=700.0))
        self.l = torch.where(D == NEG, 0.0, self.l)
        self.qo = torch.sigmoid(D)
        lse = mass.log() + torch.nn.functional.softplus(-D, threshold=700.0)
        lse = torch.where(D == NEG, self.xt - safe, lse)
        self.logq = x - safe[:, None] - lse[:, None]
        self.logq.scatter_(1, self.t[:, None], self.l[:, None])
        self.logq = torch.where(self.empty[:, None], NEG, self.logq)
        self.q = self.logq.exp()
        self.H = -torch.where(self.q == 0, 0.0, self.q * self.logq).sum(-1)
        zbar = torch.where(e > 0, e * self.z.abs(), 0.0).sum(-1) / mass.clamp(min=1e-300)
        parts = D.abs() + mass.log().abs() + (safe - self.xt).abs() + 1
        finite = torch.isfinite(parts)
        self.dm = SUM + EXP * zbar                                     # of the others' mass, relative
        self.dl = torch.where(finite, self.qo * (self.dm + 6 * STEP * parts), 0.0) + 4 * STEP * self.l.abs() + 1e-37
        self.dl = torch.where(torch.isfinite(self.dl), self.dl, 0.0)
        # a weighted sum over a sum, the logarithm of the mass, and the token's share
        self.dH = 3 * (self.dm + 6 * STEP * torch.where(finite, parts, 0.0)) * (self.H + 1) + 1e-37

    def gradient(self, a, b, scale, da=None):
        """scale d (a l + b H) / d logits and its bound; da: a's own."""
        import torch
        a, scale = a[:, None], (scale / self.tau)[:, None]
        b = torch.zeros_like(a) if b is None else b[:, None]
        surprise = torch.where(self.q == 0, 0.0, -self.logq)
        one = torch.zeros_like(self.q).scatter_(1, self.t[:, None], 1.0)
        share = torch.where(one > 0, self.qo[:, None], -self.q)         # 1[v = t] - q_v
        g = scale * (a * share + b * self.q * (surprise - self.H[:, None]))
        rel = 2 * (SUM + EXP * torch.where(self.q > 1e-40, self.z.abs(), 0.0) + self.dm[:, None])
        weight = share.abs() * a.abs() + self.q * b.abs() * (surprise + self.H[:, None])
        bound = scale.abs() * (weight * rel + self.q * b.abs() * (self.dH + self.dl)[:, None] + share.abs() * (
            0.0 if da is None else da[:, None]) + 1e-37 * (1 + a.abs() + 200 * b.abs()))
        out = (self.empty | ~self.live)[:, None]
        return torch.where(out, 0.0, g), torch.where(out, 0.0, bound)


def policy(r, A, old, ref, weight, low, high, dual, kl, bonus):
    """(loss, bound, slope in l, bound) of every row of Rows r, all in 64 bits."""
    import torch
    A = A.double()
    old = r.l if old is None else old.double()
    same = r.l == old
    gap = torch.where(same, 0.0, r.l - old)
    ratio = gap.exp()
    kept = torch.where((A == 0) & torch.isinf(ratio), 0.0, ratio * A)
    other = ratio.clamp(1 - low, 1 + high) * A
    gain = torch.minimum(kept, other)
    slope = torch.where(other < kept, 0.0, -kept)
    if dual:
        hit = (A < 0) & (gain < dual * A)
        gain, slope = torch.where(hit, dual * A, gain), torch.where(hit, 0.0, slope)
    loss = -gain
    dl = r.dl + 2 * STEP * (torch.where(torch.isfinite(gap), gap.abs(), 0.0) + 4)
    off = kept.abs() * dl
    doff = kept.abs() * dl
    if kl:
        d = torch.where(r.l == ref.double(), 0.0, ref.double() - r.l)
        loss = loss + kl * (torch.expm1(d) - d)
        slope = slope - kl * torch.expm1(d)
        dd = dl + 2 * STEP * d.abs()
        off = off + kl * (torch.expm1(d).abs() * dd + dd * dd + 8 * STEP * (torch.expm1(d) - d).abs())
        doff = doff + kl * (d.exp() * dd + 8 * STEP * torch.expm1(d).abs())
    loss = loss - bonus * r.H
    off = off + abs(bonus) * r.dH + 4 * STEP * loss.abs() + 1e-37
    out = r.empty | ~r.live | (torch.zeros_like(r.live) if weight is None else weight == 0)
    return torch.where(out, 0.0, loss), torch.where(out, 0.0, off), torch.where(out, 0.0, slope), torch.where(out, 0.0, doff)


def near(got, want, bound, half=0.0):
    """Finite values within the bound and a rounding, all others equal; what the result's type does not reach is infinite in it."""
    import torch
    want = torch.where(torch.isinf(want.to(got.dtype)), want.sign() * math.inf, want)
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not bool(torch.isinf(got[fine]).any()), "infinities"
    off = ((got - want).abs() - bound.abs() - half * want.abs())[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{float(off.max()):.3g} beyond the bound"


def sampled(logits, tau, g):
    """A token of every row by its distribution (any, where nothing has mass)."""
    import torch
    noise = -torch.log(-torch.log(torch.rand(logits.shape, generator=g, device=logits.device).clamp(1e-30, 1 - 1e-7)))
    return (logits.float() / tau + noise).argmax(-1).int()


def away(gap, low, high, by=1e-3):
    """Logarithms of ratios, moved off the clip's borders."""
    for border in (1 - low, 1 + high):
        if border > 0:
            import torch
            gap = torch.where((gap - math.log(border)).abs() < by, gap + 3 * by, gap)
    return gap
