"""The operators on rows of logits (rules, top-K lists, divergences with gradients) against their definitions in 64 bits.

Tolerances.  ex2.approx is within 2^-22; its argument (x - m) log2(e) / tau = z is built in four fp32 steps, so an exponential
is off by 2^-22 + 4 ln2 2^-24 |z| < 2.4e-7 + 1.7e-7 |z|.  A row's sums add up to 64 terms per thread in a chain and then at
most 15 merges of two factors and three roundings each: (64 + 45) 2^-24 + 15 2^-22 < 1.1e-5.  So SUM = 1.2e-5 bounds a sum's relative
error apart from its terms' z, and EXP = 2e-7 times |z| an exponential's.  z enters the tolerances as it is in 64 bits."""
import math

import numpy as np
import pytest

from paper_2608_18183_b200 import binding

pytestmark = pytest.mark.gpu

SUM, EXP, HALF = 1.2e-5, 2e-7, {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}
NEG = float("-inf")


def _t(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[name]


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(seed, rows, V, scale=3.0, dtype="fp32", pad=0, shift=0):
    """[rows, V] view with row stride V + pad whose first element lies `shift` elements into its buffer."""
    import torch
    buf = torch.randn(rows * (V + pad) + shift + 8, generator=_gen(seed), device="cuda").mul_(scale).to(_t(dtype))
    return buf[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]


# ------------------------------------------------------------------ rules on logits
def _adjust_ref(x, u=None, s=1.0, bias=None, mask=None, mask_row=None, hist=None, hrow=None, hlen=None, rho=1.0, f=0.0,
                pr=0.0):
    """(result, bound of the fp32 arithmetic's error) in 64 bits, row by row."""
    import torch
    l = x.double()
    size = l.abs()
    if u is not None:
        size = abs(s) * (l.abs() + u.double().abs()) + u.double().abs()
        l = u.double() + s * (l - u.double())
    rows, V = l.shape
    f32 = lambda y: float(np.float32(y))
    if hist is not None:
        for r in range(rows):
            h = r if hrow is None else int(hrow[r])
            if not 0 <= h < hist.shape[0]:
                continue
            m = hist.shape[1] if hlen is None else min(max(int(hlen[r]), 0), hist.shape[1])
            tok = hist[h, :m].long()
            tok = tok[(tok >= 0) & (tok < V)]
            n = torch.bincount(tok, minlength=V).double()
            pen = torch.where(l[r] > 0, l[r] / f32(rho), l[r] * f32(rho)) - n * f32(f) - f32(pr)
            l[r] = torch.where(n > 0, pen, l[r])
            size[r] = torch.where(n > 0, size[r] * max(rho, 1 / rho) + n * abs(f) + abs(pr), size[r])
    if bias is not None:
        l = l + bias.double()
        size = size + bias.double().abs()
    if mask is not None:
        words = mask.long() & 0xFFFFFFFF
        v = torch.arange(V, device=x.device)
        bit = (words[:, v // 32] >> (v % 32)) & 1
        for r in range(rows):
            m = 0 if mask_row is None else int(mask_row[r])
            if 0 <= m < mask.shape[0]:
                l[r] = l[r].masked_fill(bit[m] == 0, NEG)
    return torch.where(torch.isnan(l), NEG, l), size


def _check_adjust(x, dtype, **kw):
    import torch
    got = binding.hbsjd_adjust_logits(x, kw.get("u"), kw.get("s", 1.0), kw.get("bias"), kw.get("mask"), kw.get("mask_row"),
                                      kw.get("hist"), kw.get("hrow"), kw.get("hlen"), kw.get("rho", 1.0), kw.get("f", 0.0),
                                      kw.get("pr", 0.0), out=kw.pop("out", None))
    want, size = _adjust_ref(x, **kw)
    assert got.dtype == x.dtype and got.shape == x.shape
    g = got.double()
    assert torch.equal(torch.isinf(g), torch.isinf(want)) and not bool(torch.isnan(g).any())
    ok = torch.isfinite(want)
    # at most eight fp32 roundings of values of that size, and the result's own
    tol = 8 * HALF["fp32"] * size + HALF[dtype] * want.abs() + 1e-38
    assert bool(((g - want).abs() <= tol)[ok].all())
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(1, 0, 0), (5, 0, 0), (33, 0, 1), (1000, 3, 0), (4099, 0, 0), (8192, 0, 0),
                                         (16384, 0, 0), (20011, 0, 3), (8200, 8, 8)])
def test_adjust_every_rule(dtype, V, pad, shift):
    import torch
    rows, g = 7, _gen(V)
    x, u = _rows(1, rows, V, dtype=dtype, pad=pad, shift=shift), _rows(2, rows, V, dtype=dtype, pad=pad, shift=shift)
    words = (V + 31) // 32
    mask = torch.randint(-2 ** 31, 2 ** 31, (3, words + 2), generator=g, device="cuda").int()
    hist = torch.randint(-3, V + 3, (4, 57), generator=g, device="cuda").int()
    hist[:, ::3] = V // 2                                       # one token again and again
    hrow = torch.tensor([0, 1, 1, 3, 2, -1, 4], device="cuda").int()
    hlen = torch.tensor([57, 0, 1, 30, 99, 10, 10], device="cuda").int()
    mrow = torch.tensor([0, 1, 2, -1, 3, 1, 0], device="cuda").int()
    bias = torch.randn(V, generator=g, device="cuda")
    all_on = dict(u=u, s=3.0, bias=bias, mask=mask, mask_row=mrow, hist=hist, hrow=hrow, hlen=hlen, rho=1.3, f=0.2, pr=0.4)
    _check_adjust(x, dtype, **all_on)
    _check_adjust(x, dtype, u=u, s=-0.5)
    _check_adjust(x, dtype, bias=bias)
    _check_adjust(x, dtype, mask=mask)
    _check_adjust(x, dtype, hist=hist, hrow=hrow, rho=0.7)
    _check_adjust(x, dtype, hist=hist, hrow=hrow, hlen=hlen, f=-0.3)
    plain = _check_adjust(x, dtype)
    assert torch.equal(plain, x)                                # no rule: the same bits
    # rows that are aligned otherwise than the output's
    _check_adjust(x, dtype, **dict(all_on, u=_rows(2, rows, V, dtype=dtype, pad=pad + 1, shift=shift + 1)))
    # in place, and over the second branch
    want = _check_adjust(x, dtype, **all_on)
    y = x.clone() if pad == 0 else x
    assert binding.hbsjd_adjust_logits(y, u, 3.0, bias, mask, mrow, hist, hrow, hlen, 1.3, 0.2, 0.4, out=y) is y
    assert torch.equal(y, want)


def test_adjust_masked_branches_infinities_and_nan():
    import torch
    x, u = _rows(3, 6, 300), _rows(4, 6, 300)
    x[0], u[0] = NEG, NEG                                       # a row that is masked in both branches
    x[1, ::2], u[1, ::2] = NEG, NEG
    x[2, 5] = float("nan")
    x[3], u[3] = torch.finfo(torch.float32).min, 0.0            # the type's lowest value
    x[4, 7], u[4, 8] = NEG, NEG
    bias = torch.zeros(300, device="cuda")
    bias[9] = NEG
    got = binding.hbsjd_adjust_logits(x, u, 2.0, bias)
    want = (u.double() + 2.0 * (x.double() - u.double()) + bias.double()).float()
    want = torch.where(torch.isnan(want), NEG, want)
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    assert bool((got[0] == NEG).all()) and got[2, 5] == NEG and bool((got[:, 9] == NEG).all())
    # a mask that leaves nothing
    none = torch.zeros(1, 10, dtype=torch.int32, device="cuda")
    assert bool((binding.hbsjd_adjust_logits(x, mask=none) == NEG).all())


def test_adjust_long_history_and_many_rows():
    """A history much longer than the vocabulary (counts above 16 bits), and more rows than a launch has CTAs at once."""
    import torch
    hist = torch.zeros(1, 100000, dtype=torch.int32, device="cuda")
    hist[0, ::10] = 3
    x = torch.zeros(1, 8, device="cuda")
    got = binding.hbsjd_adjust_logits(x, history=hist, frequency=1.0)
    assert got[0, 0] == -90000.0 and got[0, 3] == -10000.0 and bool((got[0, [1, 2, 4, 5, 6, 7]] == 0).all())
    x = _rows(5, 5000, 130)
    hist = torch.randint(0, 130, (5000, 40), generator=_gen(6), device="cuda").int()
    _check_adjust(x[:300], "fp32", hist=hist[:300], rho=2.0, pr=1.0)
    full = binding.hbsjd_adjust_logits(x, history=hist, repetition=2.0, presence=1.0)
    assert torch.equal(full[:300], binding.hbsjd_adjust_logits(x[:300], history=hist[:300], repetition=2.0, presence=1.0))


# ------------------------------------------------------------------ top-K lists
def _topk_ref(x, k, tau):
    import torch
    l = torch.where(torch.isnan(x), NEG, x.double())
    v, i = torch.sort(l, dim=-1, descending=True, stable=True)
    rest = torch.logsumexp(v[:, k:] / tau, -1) if k < x.shape[1] else torch.full_like(v[:, 0], NEG)
    return v[:, :k], torch.where(v[:, :k] == NEG, -1, i[:, :k]), rest


def _check_topk(x, k, tau=1.0):
    import torch
    values, indices, rest = binding.hbsjd_topk_logits(x, k, temperature=tau)
    v, i, r = _topk_ref(x, k, tau)
    assert torch.equal(indices.long(), i)
    assert torch.equal(values.double(), v)
    inf = torch.isinf(r)
    assert torch.equal(rest.double()[inf], r[inf])
    ok = ~inf
    # the sum's error, its terms' (those near the largest of the rest weigh: |z| <= 60), and the roundings of m / tau and the sum
    tol = SUM + EXP * 60 + 4 * HALF["fp32"] * (r.abs() + (x.double().nan_to_num(0, 0, 0).abs().amax(-1) / tau))
    assert bool(((rest.double() - r).abs() <= tol)[ok].all()), float(((rest.double() - r).abs() - tol)[ok].max())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,k,rows,pad,shift", [
    (1, 1, 3, 0, 0), (7, 3, 5, 0, 1), (64, 64, 4, 0, 0), (100, 1, 600, 1, 0), (1000, 8, 40, 0, 0), (1000, 999, 3, 0, 0),
    (1025, 64, 300, 0, 5), (2048, 256, 200, 0, 0), (4099, 1024, 31, 0, 0), (5000, 300, 17, 24, 8), (16384, 64, 700, 0, 0),
    (16384, 1024, 160, 0, 0), (16384, 1, 2, 0, 0), (16384, 512, 9, 0, 0), (20011, 130, 30, 0, 0), (32768, 256, 90, 0, 0),
    (65537, 64, 20, 0, 0), (131072, 1024, 3, 0, 0)])
def test_topk_shapes(dtype, V, k, rows, pad, shift):
    x = _rows(V + k, rows, V, 3.5, dtype, pad, shift)
    _check_topk(x, k)
    _check_topk(x, k, 0.6)


@pytest.mark.parametrize("V,k", [(16384, 64), (16384, 700), (20000, 64), (1500, 100), (65536, 50)])
def test_topk_orders_that_crowd(V, k):
    """Rows whose largest entries do not spread: sorted either way, in a few threads' groups only, ties of every extent, masks by
    -inf and by the lowest value, NaN, infinities, adjacent floats, +0 and -0, denormals, a rest far below."""
    import torch
    g = _gen(V)
    base = torch.randn(V, generator=g, device="cuda") * 3
    low = torch.finfo(torch.float32).min
    up = base.sort().values
    rows = [up, up.flip(0), torch.zeros(V, device="cuda"), base.round(), torch.full((V,), NEG, device="cuda"),
            torch.full((V,), low, device="cuda"), torch.full((V,), float("nan"), device="cuda")]
    for few in (1, k - 1, k, k + 1, 5 * k):
        for value in (NEG, low, float("nan")):
            r = torch.full((V,), value, device="cuda")
            at = torch.randperm(V, generator=g, device="cuda")[:few]
            r[at] = base[at]
            rows.append(r)
    for stride in (64, 512, 1024, 2048, 4096):                 # the largest all lie in the same groups
        r = base.clone()
        r[::stride] += 100
        rows.append(r)
        r = base.clone()
        r.view(-1)[(torch.arange(V, device="cuda") // 4) % (stride // 4) < 2] += 50
        rows.append(r)
    r = base.clone()
    r[: k // 2 + 1] = float("inf")
    rows.append(r)
    rows.append(1.0 + torch.arange(V, device="cuda") * 2.0 ** -23)
    rows.append(torch.where(base > 0, 0.0, -0.0))
    rows.append(base * 1e-42)
    r = torch.full((V,), -500.0, device="cuda")
    r[5:5 + k] = 30 + base[5:5 + k]                            # the rest is e^-500 of the list
    rows.append(r)
    r = torch.full((V,), 2.0, device="cuda")
    r[V // 3:V // 3 + k // 2] = 7.0                            # the k-th is one of very many
    rows.append(r)
    x = torch.stack(rows)
    _check_topk(x, k)
    _check_topk(x.bfloat16(), k, 2.0)
    one = torch.cat([x] * 12)                                  # the same rows where no row is split over CTAs
    _check_topk(one, k)
    a, b = binding.hbsjd_topk_logits(one, k), binding.hbsjd_topk_logits(x, k)
    assert all(torch.equal(p[:len(x)], q) for p, q in zip(a[:2], b[:2]))


# ------------------------------------------------------------------ divergences
def _masked_log_softmax(x):
    """log softmax and softmax in 64 bits, against the row's largest (a row of the lowest value is uniform); rows without
    mass are -inf and 0."""
    import torch
    m = x.amax(-1, keepdim=True)
    x = x - torch.where(m == NEG, 0.0, m)
    l = torch.log(torch.exp(x).sum(-1, keepdim=True))
    l = torch.where(l == NEG, 0.0, l)
    return x - l, torch.exp(x - l)


def _distill_ref(s, t, w, tau, a, b, least=2.0 ** -126):
    """loss, gradient and bounds of their errors, in 64 bits."""
    import torch
    lq, q = _masked_log_softmax(s.double() / tau)
    lp, p = _masked_log_softmax(t.double() / tau)
    q, p = torch.where(q < least, 0.0, q), torch.where(p < least, 0.0, p)
    r = lq - lp
    F = torch.where(p > 0, -p * r, 0.0).sum(-1, keepdim=True)
    R = torch.where(q > 0, q * r, 0.0).sum(-1, keepdim=True)
    none = ((q.sum(-1) == 0) | (p.sum(-1) == 0))[:, None]
    W = w.double()[:, None]
    dead = none | (W == 0)
    loss = (a * F if a else 0.0) + (b * R if b else 0.0)
    rev = torch.where(q > 0, q * (r - R), 0.0) if b else torch.zeros_like(q)
    grad = (a * (q - p) + b * rev) * W / tau
    # logarithms of masses are off by SUM + EXP |z|, d by the roundings of both its parts, which are about |z|
    fin = lambda v: torch.where(torch.isfinite(v), v.abs(), 0.0)
    zq, zp = fin(lq), fin(lp)
    d = torch.where((q > 0) | (p > 0), torch.minimum(zq, fin(r) + zp) + torch.minimum(zp, fin(r) + zq), 0.0)
    eq, ep = (q * d).sum(-1, keepdim=True), (p * d).sum(-1, keepdim=True)
    zm = torch.maximum((q * zq).sum(-1, keepdim=True), (p * zp).sum(-1, keepdim=True))
    rel = 2 * SUM + EXP * (zm + 10)
    tl = (a + b) * rel * (eq + ep + 1)
    tg = (a * (q * (rel + EXP * zq) + p * (rel + EXP * zp)) + b * q * (rel + EXP * zq) * (d + eq + 1)) * W.abs() / tau
    zero = lambda v: torch.where(dead, 0.0, v)
    return zero(loss)[:, 0], zero(grad), tl[:, 0] + 1e-37, tg + 1e-37


def _compare(loss, grad, ref, dtype):
    import torch
    rl, rg, tl, tg = ref
    l = loss.double()
    assert torch.equal(torch.isnan(l), torch.isnan(rl)), (l, rl)
    assert torch.equal(torch.isinf(l), torch.isinf(rl)), (l, rl)
    ok = torch.isfinite(rl)
    assert bool(((l - rl).abs() <= tl + HALF["fp32"] * rl.abs())[ok].all()), float(((l - rl).abs() / tl)[ok].max())
    if grad is not None:
        g = grad.double()
        ok = torch.isfinite(rg)
        assert bool(torch.isfinite(g)[ok].all())
        err, tol = (g - rg).abs(), tg + HALF[dtype] * rg.abs()
        assert bool((err <= tol)[ok].all()), float((err / tol)[ok].max())


@pytest.mark.parametrize("ds,dt", [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("V,rows,pad,shift", [
    (1, 3, 0, 0), (6, 5, 0, 1), (129, 200, 0, 0), (1000, 40, 3, 0), (4096, 300, 0, 0), (5003, 9, 0, 2), (16384, 160, 0, 0),
    (16384, 3, 0, 0), (20011, 33, 0, 0), (36864, 5, 8, 8), (65537, 90, 0, 0), (131072, 4, 0, 0)])
def test_distill_shapes(ds, dt, V, rows, pad, shift):
    import torch
    s = _rows(V, rows, V, 3.0, ds, pad, shift)
    t = (_rows(V + 1, rows, V, 2.0, dt, pad, shift).float() + 0.6 * s.float()).to(_t(dt))
    w = torch.rand(rows, generator=_gen(V), device="cuda")
    w[::3] = 0
    for tau, a, b in ((1.0, 0.5, 0.5), (0.7, 1.0, 0.0), (2.0, 0.0, 1.0), (1.0, 0.3, 0.9)):
        ref = _distill_ref(s, t, w, tau, a, b)
        loss, grad = binding.hbsjd_distill(s, t, w, tau, a, b)
        assert grad.dtype == s.dtype and grad.shape == s.shape
        _compare(loss, grad, ref, ds)
        assert bool((loss[::3] == 0).all()) and bool((grad[::3] == 0).all())
        only, none = binding.hbsjd_distill(s, t, w, tau, a, b, want_grad=False)
        assert none is None and torch.equal(only, loss)
    # rows whose arrays are aligned in three ways, and the gradient over the student's or the teacher's logits
    t2, g2 = _rows(0, rows, V, 1.0, dt, pad + 1, shift + 1), _rows(0, rows, V, 1.0, ds, pad + 2, shift + 1)
    t2.copy_(t)
    loss, grad = binding.hbsjd_distill(s, t2, w, grad=g2)
    assert grad is g2
    _compare(loss, grad, _distill_ref(s, t, w, 1.0, 0.5, 0.5), ds)
    for over in (s, t) if ds == dt else (s,):
        a, b = s.clone(), t.clone()
        over = a if over is s else b
        want = binding.hbsjd_distill(a, b, w)                   # (how a row is aligned decides the order of its sums)
        loss, grad = binding.hbsjd_distill(a, b, w, grad=over)
        assert torch.equal(loss, want[0])
        _compare(loss, grad, _distill_ref(s, t, w, 1.0, 0.5, 0.5), ds)


def _buckets(s, values, indices, rest):
    """Teacher and student as 64-bit logits over the whole vocabulary from a list: what the first valid entries of a row say."""
    rows, V = s.shape
    listed = []
    for r in range(rows):
        seen = {}
        for v, i in zip(values[r].tolist(), indices[r].tolist()):
            if 0 <= i < V and v != NEG and i not in seen:
                seen[i] = v
        listed.append(seen)
    return listed


def _distill_topk_ref(s, values, indices, rest, w, tau, a, b):
    """Reference through the k + 1 outcomes: the listed tokens' logits and the log mass of all others, as logits at tau = 1."""
    import torch
    rows, V = s.shape
    listed = _buckets(s, values, indices, rest)
    k = max([len(x) for x in listed] + [1])
    S = torch.full((rows, k + 1), NEG, dtype=torch.float64, device="cuda")
    T = S.clone()
    where = torch.zeros(rows, k, dtype=torch.long, device="cuda")
    other = torch.ones(rows, V, dtype=torch.bool, device="cuda")
    x = s.double() / tau
    x = x - torch.nan_to_num(x.amax(-1, keepdim=True), neginf=0.0)  # (of a row of the lowest value 64 bits would keep nothing else)
    for r, seen in enumerate(listed):
        if seen:
            at = torch.tensor(list(seen), device="cuda")
            where[r, :len(seen)] = at
            S[r, :len(seen)] = x[r, at]
            T[r, :len(seen)] = torch.tensor(list(seen.values()), dtype=torch.float64, device="cuda") / tau
            other[r, at] = False
    xo = torch.where(other, x, NEG)
    S[:, k] = torch.logsumexp(xo, -1)
    if rest is not None:
        T[:, k] = rest.double()
    loss, g, tl, tg = _distill_ref(S, T, w, 1.0, a, b)
    share = torch.exp(xo - torch.where(S[:, k:] == NEG, 0.0, S[:, k:]))
    # (the share's own error: a sum's and an exponential's)
    z = torch.where(torch.isfinite(xo - S[:, k:]), (xo - S[:, k:]).abs(), 0.0)
    grad, tol = g[:, k:] * share / tau, tg[:, k:] * share / tau
    grad = torch.where(share == 0, 0.0, grad)
    tol = tol + grad.abs() * (2 * SUM + EXP * z) + 1e-37       # (shares below 2^-126 = 1.2e-38 are none)
    for r, seen in enumerate(listed):
        n = len(seen)
        grad[r, where[r, :n]] = g[r, :n] / tau
        tol[r, where[r, :n]] = tg[r, :n] / tau
    # the rest is given as a logarithm: it and its difference from the largest listed logit are rounded by its size
    if rest is not None:
        big = torch.where(torch.isfinite(T), T.abs(), 0.0).amax(-1)
        big = torch.where(big < 1e30, big, 0.0)
        tl = tl + (a + b) * 8 * HALF["fp32"] * big
        tol = tol + 8 * HALF["fp32"] * (big * w.abs())[:, None] / tau * (a + b) * _masked_log_softmax(x)[1]
    return loss, grad, tl, tol


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,k,rows,pad,shift", [
    (1, 1, 3, 0, 0), (9, 9, 4, 0, 1), (100, 7, 50, 1, 0), (1000, 1, 20, 0, 0), (1000, 1000, 3, 0, 0), (2050, 64, 90, 0, 3),
    (8192, 300, 20, 0, 0), (16384, 64, 160, 0, 0), (16384, 64, 3, 0, 0), (20011, 1024, 30, 0, 0), (32768, 32, 9, 8, 8),
    (65537, 128, 80, 0, 0), (131072, 512, 3, 0, 0)])
def test_distill_topk_shapes(dtype, V, k, rows, pad, shift):
    import torch
    s = _rows(V, rows, V, 3.0, dtype, pad, shift)
    t = _rows(V + 1, rows, V, 2.0) + 0.6 * s.float()
    w = torch.rand(rows, generator=_gen(V), device="cuda")
    w[1::3] = 0
    for tau, a, b, with_rest in ((1.0, 0.5, 0.5, True), (0.7, 1.0, 0.0, True), (2.0, 0.0, 1.0, True), (1.0, 1.0, 0.0, False)):
        values, indices, rest = binding.hbsjd_topk_logits(t, k, temperature=tau)
        rest = rest if with_rest else None
        ref = _distill_topk_ref(s, values, indices, rest, w, tau, a, b)
        loss, grad = binding.hbsjd_distill_topk(s, values, indices, rest, w, tau, a, b)
        assert grad.dtype == s.dtype
        _compare(loss, grad, ref, dtype)
        assert bool((loss[1::3] == 0).all()) and bool((grad[1::3] == 0).all())
        only, none = binding.hbsjd_distill_topk(s, values, indices, rest, w, tau, a, b, want_grad=False)
        assert none is None and torch.equal(only, loss)
    values, indices, rest = binding.hbsjd_topk_logits(t, k)
    g2 = _rows(0, rows, V, 1.0, dtype, pad + 1, shift + 1)
    loss, grad = binding.hbsjd_distill_topk(s, values, indices, rest, w, grad=g2)
    _compare(loss, grad, _distill_topk_ref(s, values, indices, rest, w, 1.0, 1.0, 0.0), dtype)
    x = s.clone()
    want = binding.hbsjd_distill_topk(x, values, indices, rest, w)
    loss, grad = binding.hbsjd_distill_topk(x, values, indices, rest, w, grad=x)
    assert grad is x and torch.equal(loss, want[0])
    _compare(loss, grad, _distill_topk_ref(s, values, indices, rest, w, 1.0, 1.0, 0.0), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heavy", [False, True])
def test_divergences_that_are_small_keep_their_digits(dtype, heavy):
    """A listed token of little mass, or of all but a little.  The loss moves with the logarithms rx, ry of the listed mass over the others'
    by q_l q_o (rx - ry) drx + (p_l - q_l) dry for KL(q || p), and with the names changed for KL(p || q), however large they are;
    rx is off by what its mass is (SUM) and by the roundings of its logits, its logarithm and the rest (10 halves of its
    parts, none larger than the row's largest logits' size in temperatures, the teacher's rest and log V = 11)."""
    import torch
    V, rows, tau = 50021, 24, 2.0
    s = _rows(V, rows, V, 1.0, dtype)
    at = (torch.arange(rows, device="cuda") * 1999 + 7)
    s[torch.arange(rows, device="cuda"), at] = (torch.linspace(-6, 4, rows, device="cuda") + (38 if heavy else 0)).to(s.dtype)
    values = s.float().gather(1, at[:, None]) + torch.where(torch.arange(rows, device="cuda") % 2 == 0, 1.5, -1.5)[:, None]
    x = s.double() / tau
    xl = x.gather(1, at[:, None])[:, 0]
    xo = torch.logsumexp(x.scatter(1, at[:, None], NEG), -1)
    rest = (xo + 0.25).float()
    yl, yo = values[:, 0].double() / tau, rest.double()
    rx, ry = xl - xo, yl - yo
    lql, lqo, lpl, lpo = (torch.nn.functional.logsigmoid(v) for v in (rx, -rx, ry, -ry))
    ql, qo, pl, po = lql.exp(), lqo.exp(), lpl.exp(), lpo.exp()
    # sum f log(f / g) as a sum of terms that are none below 0: 64 bits keep all that is asked for
    kl = lambda f, lf, g, lg: sum(a * (b - d) - a + c for a, b, c, d in zip(f, lf, g, lg))
    F, R = kl((pl, po), (lpl, lpo), (ql, qo), (lql, lqo)), kl((ql, qo), (lql, lqo), (pl, po), (lpl, lpo))
    size = torch.stack([xl.abs(), xo.abs(), yl.abs(), yo.abs()]).amax(0) + 11
    dr = SUM + 10 * HALF["fp32"] * size
    dif, mass = (rx - ry).abs(), (pl - ql).abs()
    tF, tR = dr * (pl * po * dif + mass), dr * (ql * qo * dif + mass)
    # the listed token's term is its mass times a sum of logarithms, the others' theirs times one that is about the listed mass
    term = lambda f: 8 * HALF["fp32"] * f * (dif + size)
    for a, b, want, tol in ((1.0, 0.0, F, tF + term(pl)), (0.0, 1.0, R, tR + term(ql))):
        loss, _ = binding.hbsjd_distill_topk(s, values, at[:, None].int(), rest, None, tau, a, b)
        assert bool(((loss.double() - want).abs() <= tol).all()), ((loss.double() - want) / tol, want)
        if not heavy:
            assert float((tol / want).max()) < 1e-3              # (differences of logarithms near 11 would be off by 1e-6, of 1e-7 to 1e-4)


def test_distill_topk_lists_with_gaps_and_repeats():
    """Entries that count for nothing (-inf, tokens outside the vocabulary, tokens listed before), lists without an entry, in
    rows held by one CTA and by several."""
    import torch
    for V, rows in ((500, 12), (16384, 12), (16384, 320)):
        k = 40
        s = _rows(V, rows, V)
        values = torch.randn(rows, k, generator=_gen(1), device="cuda") * 2
        indices = torch.randint(0, V, (rows, k), generator=_gen(2), device="cuda").int()
        rest = torch.randn(rows, generator=_gen(3), device="cuda")
        indices[0, 5:] = -1
        indices[1, ::2] = V
        indices[2, 1:] = indices[2, 0]                          # one token forty times
        indices[3, 20:] = indices[3, :20]
        values[4, ::3] = NEG
        values[5] = NEG                                         # all of the teacher's mass is the rest
        indices[6] = 2 ** 31 - 1
        rest[6] = NEG                                           # a teacher without mass
        indices[7, 7], indices[7, 9] = -2 ** 31, V - 1
        values[8, 0], indices[8, 1] = NEG, indices[8, 0]        # the first entry of a token is void, the second counts
        rest[9] = -300.0
        w = torch.ones(rows, device="cuda")
        for a, b in ((1.0, 0.0), (0.5, 0.5)):
            got = binding.hbsjd_distill_topk(s, values, indices, rest, None, 1.0, a, b)
            _compare(*got, _distill_topk_ref(s, values, indices, rest, w, 1.0, a, b), "fp32")
        got = binding.hbsjd_distill_topk(s, values, indices, None)
        _compare(*got, _distill_topk_ref(s, values, indices, None, w, 1.0, 1.0, 0.0), "fp32")
        assert got[0][6] == 0 and bool((got[1][6] == 0).all())


def _masks(V, rows):
    """Student and teacher rows as masks leave them."""
    import torch
    low = torch.finfo(torch.float32).min
    s, t = _rows(11, rows, V), _rows(12, rows, V, 2.0)
    hide = torch.rand(rows, V, generator=_gen(13), device="cuda") < 0.5
    hide[:, 0] = False
    s[0][hide[0]], t[0][hide[0]] = NEG, NEG                     # the same mask
    s[1][hide[1]], t[1][hide[1]] = low, low
    s[2] = NEG                                                  # nothing left
    t[3] = NEG
    s[4], t[4] = NEG, NEG
    s[5] = low                                                  # uniform
    s[6], t[6] = low, low
    t[7][hide[7]] = NEG                                         # a mask on the teacher only: KL(q || p) is infinite
    s[8][hide[8]] = NEG                                         # on the student only: KL(p || q) is
    s[9, 1:], t[9, 1:] = NEG, NEG                               # one entry left
    s[10] += 1000.0
    t[11] -= 1000.0
    s[12], t[12] = t[12].clone(), t[12].clone()                 # equal rows
    s[13, 3] = float("nan")
    t[14, 4] = float("nan")
    s[15, 5] = float("inf")
    s[16, 6], t[16, 7] = 90.0, 90.0                             # nearly one-hot, and they disagree
    return s, t


@pytest.mark.parametrize("V,rows", [(257, 20), (16384, 20), (16384, 200)])
def test_distill_masks_infinities_and_nan(V, rows):
    import torch
    s, t = _masks(V, rows)
    w = torch.full((rows,), 0.5, device="cuda")
    for a, b in ((1.0, 0.0), (0.0, 1.0), (0.5, 0.5)):
        loss, grad = binding.hbsjd_distill(s, t, w, 1.0, a, b)
        rl, rg, tl, tg = _distill_ref(s, t, w, 1.0, a, b)
        for r in (13, 14, 15):
            rl[r], rg[r] = float("nan"), float("nan")
            assert bool(torch.isnan(grad[r]).all())
        if b == 0:                                              # q - p, though the loss is infinite
            assert loss[8] == float("inf")
            rg[8] = torch.where(s[8] == NEG, 0.0, torch.softmax(s[8].double(), -1)) - torch.softmax(t[8].double(), -1)
            rg[8] *= 0.5
        _compare(loss, grad, (rl, rg, tl, tg), "fp32")
        for r in (2, 3, 4):
            assert loss[r] == 0 and bool((grad[r] == 0).all())
        assert loss[12] == 0 and loss[9] == 0
    # left out rows are not read
    w[13:16] = 0
    loss, grad = binding.hbsjd_distill(s, t, w)
    assert bool((loss[13:16] == 0).all()) and bool((grad[13:16] == 0).all())


def test_distill_topk_masks_infinities_and_nan():
    import torch
    for V, rows in ((257, 20), (16384, 20), (16384, 200)):
        s, t = _masks(V, rows)
        values, indices, rest = binding.hbsjd_topk_logits(t.nan_to_num(0.0, neginf=NEG), 30)
        w = torch.ones(rows, device="cuda")
        values[14, 2] = float("nan")
        for a, b in ((1.0, 0.0), (0.5, 0.5)):
            loss, grad = binding.hbsjd_distill_topk(s, values, indices, rest, w, 1.0, a, b)
            clean = values.clone()
            clean[14, 2] = 0.0
            rl, rg, tl, tg = _distill_topk_ref(s.nan_to_num(0.0, neginf=NEG, posinf=0.0), clean, indices, rest, w, 1.0, a, b)
            for r in (13, 14, 15):
                rl[r], rg[r] = float("nan"), float("nan")
                assert bool(torch.isnan(grad[r]).all())
            if b == 0:
                rg[8] = float("inf")                            # (checked below)
            _compare(loss, grad, (rl, rg, tl, tg), "fp32")
            for r in (2, 3, 4):
                assert loss[r] == 0 and bool((grad[r] == 0).all())
            if b == 0:
                q = torch.softmax(s[8].double(), -1)
                total = torch.logsumexp(torch.cat([values[8], rest[8:9]]).double(), -1)
                at = indices[8].long()
                want = q[at] - torch.exp(values[8].double() - total)
                assert loss[8] == float("inf") and bool(((grad[8][at].double() - want).abs() < 3e-5).all())


def test_a_teacher_s_nan_shows_wherever_it_stands():
    """NaN among the listed values, also alone in its part of the row and where the student has no mass."""
    import torch
    for V, rows in ((700, 40), (16384, 200)):
        s = _rows(1, rows, V)
        values = torch.randn(rows, 12, generator=_gen(2), device="cuda")
        indices = torch.stack([torch.randperm(V, generator=_gen(3 + r), device="cuda")[:12] for r in range(rows)]).int()
        rest = torch.zeros(rows, device="cuda")
        clean = binding.hbsjd_distill_topk(s, values, indices, rest, forward=0.5, reverse=0.5)
        values[::2, 5] = float("nan")
        s[::2].scatter_(1, indices[::2, 5:6].long(), NEG)
        loss, grad = binding.hbsjd_distill_topk(s, values, indices, rest, forward=0.5, reverse=0.5)
        assert bool(torch.isnan(loss[::2]).all()) and bool(torch.isnan(grad[::2]).all())
        assert torch.equal(loss[1::2], clean[0][1::2]) and torch.equal(grad[1::2], clean[1][1::2])


def test_lists_of_one_again_and_again():
    """k = 1 leaves the selection one candidate; thousands of such rows per CTA, in rows of one CTA and of several."""
    import torch
    for V, rows in ((40, 9000), (1200, 9000), (5000, 6000), (90000, 300)):
        x = _rows(V, rows, V)
        for _ in range(3):
            values, indices, rest = binding.hbsjd_topk_logits(x, 1)
            m = x.max(-1)
            assert torch.equal(values[:, 0], m.values) and torch.equal(indices[:, 0].long(), m.indices)


def test_a_list_of_everything_is_the_whole_divergence():
    import torch
    s, t = _rows(1, 9, 1000), _rows(2, 9, 1000)
    full = binding.hbsjd_distill(s, t, temperature=1.5, forward=0.4, reverse=0.6)
    listed = binding.hbsjd_distill_topk(s, *binding.hbsjd_topk_logits(t, 1000, 1.5), None, 1.5, 0.4, 0.6)
    assert bool(((full[0] - listed[0]).abs() <= 4 * SUM * (1 + full[0].abs())).all())
    assert bool(((full[1] - listed[1]).abs() <= 4 * SUM * (full[1].abs() + 1e-3)).all())


@pytest.mark.parametrize("entry", ["distill", "topk"])
def test_gradients_against_differences(entry):
    """Central differences of the loss in 64 bits would test the reference; here the kernel's own loss is differenced along random
    directions.  The loss is good to SUM (1 + loss); h = 0.05 along a direction of unit size leaves an error of h^2 / 6 times
    the third derivative, below 1 there, and 2 SUM (1 + loss) / 2h: 4.2e-4 + 2.4e-4 (1 + loss)."""
    import torch
    rows, V, h = 6, 600, 0.05
    s, t = _rows(1, rows, V, 1.5), _rows(2, rows, V, 1.5)
    lists = binding.hbsjd_topk_logits(t, 20)

    def f(x):
        if entry == "distill":
            return binding.hbsjd_distill(x, t, forward=0.7, reverse=0.6)
        return binding.hbsjd_distill_topk(x, *lists, forward=0.7, reverse=0.6)

    loss, grad = f(s)
    g = _gen(5)
    for _ in range(8):
        d = torch.randn(rows, V, generator=g, device="cuda")
        d[:, ::2] *= 4
        d /= d.norm(dim=-1, keepdim=True)
        up, down = f(s + h * d)[0].double(), f(s - h * d)[0].double()
        want = (up - down) / (2 * h)
        got = (grad.double() * d.double()).sum(-1)
        assert bool(((got - want).abs() <= 4.2e-4 + 2.4e-4 * (1 + loss)).all())


def test_distill_is_the_score_s_divergence():
    """At the defaults the loss is what hbsjd_bikl computes."""
    from paper_2608_18183_b200 import synth
    import torch
    sh = synth.ModelShape(1, 64, 1, 64, 16384, 4, 4, 3, "bf16")
    ctx = binding.Context(sh, synth.make_weights(sh, 3, target_entropy=None), 2, 4)
    s, t = _rows(1, 300, 16384), _rows(2, 300, 16384)
    a, b = ctx.hbsjd_bikl(s, t), binding.hbsjd_distill(s, t, want_grad=False)[0]
    assert bool(((a - b).abs() <= 4 * SUM * (1 + a)).all())
    ctx.hbsjd_destroy()


# ------------------------------------------------------------------ calls
def test_rows_beyond_32_bits():
    """Rows whose offsets pass 2^31 elements: the last rows are as they are alone, and rows between the strides stay."""
    import torch
    V, ld, rows = 1000, 1 << 20, 2500
    buf = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(rows, ld)[:, :V]
    x.copy_(_rows(1, rows, V, dtype="bf16"))
    t = _rows(2, rows, V, dtype="bf16")
    # (the number of rows decides how many threads sum over one: two sums, each within SUM + EXP |z| of the same value)
    a, b = binding.hbsjd_topk_logits(x, 20), binding.hbsjd_topk_logits(x[-30:].contiguous(), 20)
    assert torch.equal(a[0][-30:], b[0]) and torch.equal(a[1][-30:], b[1])
    assert bool(((a[2][-30:] - b[2]).abs() <= 2 * (SUM + EXP * 60)).all())
    want = binding.hbsjd_distill(x[-30:].contiguous(), t[-30:])
    adjusted = binding.hbsjd_adjust_logits(x[-30:].contiguous(), bias=torch.ones(V, device="cuda"))
    got = binding.hbsjd_distill(x, t, grad=x)
    assert torch.equal(got[0][-30:], want[0]) and torch.equal(got[1][-30:], want[1])
    assert not bool(buf.view(rows, ld)[:, V:].any())
    x.copy_(_rows(1, rows, V, dtype="bf16"))
    binding.hbsjd_adjust_logits(x, bias=torch.ones(V, device="cuda"), out=x)
    assert torch.equal(x[-30:], adjusted)


def _all_four(s, t, bias, history, stream=None):
    x = binding.hbsjd_adjust_logits(s, bias=bias, repetition=1.5, history=history, stream=stream)
    lists = binding.hbsjd_topk_logits(t, 16, stream=stream)
    return (x, *lists, *binding.hbsjd_distill_topk(x, *lists, forward=0.5, reverse=0.5, stream=stream),
            *binding.hbsjd_distill(x, t, stream=stream))


def test_streams_graphs_and_repeats():
    """The same bits from every call: again, on another stream, at the same time on two, and replayed from a graph on new
    contents."""
    import torch
    for rows, V in ((3, 16384), (200, 5003)):
        s, t = _rows(1, rows, V), _rows(2, rows, V)
        side = torch.full((V,), 0.25, device="cuda"), torch.zeros(rows, 3, dtype=torch.int32, device="cuda")
        want = _all_four(s, t, *side)
        same = lambda got: all(torch.equal(a, b) for a, b in zip(got, want))
        for _ in range(3):
            assert same(_all_four(s, t, *side))
        one, two = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        a = [_all_four(s, t, *side, st) for st in (one, two, one, two)]
        torch.cuda.synchronize()
        assert all(same(x) for x in a)
        with torch.cuda.stream(one):
            x = _all_four(s, t, *side)
        torch.cuda.synchronize()
        assert same(x)
        s2, t2 = torch.zeros_like(s), torch.zeros_like(t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = _all_four(s2, t2, *side)
        for _ in range(2):
            s2.copy_(s)
            t2.copy_(t)
            graph.replay()
            torch.cuda.synchronize()
            assert same(out)
            s2.zero_()
            t2.zero_()
        del graph


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,rows", [(40001, 700), (100000, 300), (7, 70000), (2500, 5000)])
def test_many_rows_of_every_length(dtype, V, rows):
    """More rows than clusters or CTAs run at once, so that each takes several, of both kinds: in work and left out."""
    import torch
    s, t = _rows(1, rows, V, 3.0, dtype), _rows(2, rows, V, 2.0, dtype)
    w = torch.rand(rows, generator=_gen(3), device="cuda")
    w[torch.rand(rows, generator=_gen(4), device="cuda") < 0.4] = 0
    k = min(V, 50)
    _check_topk(t, k)
    lists = binding.hbsjd_topk_logits(t, k)
    some = torch.randperm(rows, generator=_gen(5), device="cuda")[:60].sort().values
    loss, grad = binding.hbsjd_distill_topk(s, *lists, w, 1.0, 0.5, 0.5)
    ref = _distill_topk_ref(s[some], *(x[some] for x in lists), w[some], 1.0, 0.5, 0.5)
    _compare(loss[some], grad[some], ref, dtype)
    assert bool((loss[w == 0] == 0).all()) and not bool(grad[w == 0].any())
    full = binding.hbsjd_distill(s, t, w, 1.0, 0.5, 0.5)
    _compare(full[0][some], full[1][some], _distill_ref(s[some], t[some], w[some], 1.0, 0.5, 0.5), dtype)
    assert bool((full[0][w == 0] == 0).all()) and not bool(full[1][w == 0].any())
    # every other row against a call of its own, which deals the rows otherwise: twice the tolerance of one
    half = slice(1, None, 2)
    again = binding.hbsjd_distill(s[half].contiguous(), t[half].contiguous(), w[half].contiguous(), 1.0, 0.5, 0.5)
    size = (s.double() - t.double()).abs().amax() + 20
    assert bool(((again[0] - full[0][half]).abs() <= 4 * (SUM + EXP * 60) * size).all())
    assert torch.equal(binding.hbsjd_adjust_logits(s, bias=torch.zeros(V, device="cuda")), s)


def test_two_host_threads_at_once():
    import threading
    import torch
    rows, V = 300, 9001
    s, t = _rows(1, rows, V), _rows(2, rows, V)
    side = torch.full((V,), 0.25, device="cuda"), torch.zeros(rows, 3, dtype=torch.int32, device="cuda")
    want = _all_four(s, t, *side)
    torch.cuda.synchronize()
    bad = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = _all_four(s, t, *side)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    bad.append(1)
        stream.synchronize()

    threads = [threading.Thread(target=work) for _ in range(3)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not bad


def test_masks_of_unsigned_words():
    import torch
    x = _rows(1, 3, 100)
    mask = torch.randint(-2 ** 31, 2 ** 31, (2, 4), generator=_gen(2), device="cuda").int()
    row = torch.tensor([0, 1, 1], device="cuda").int()
    assert torch.equal(binding.hbsjd_adjust_logits(x, mask=mask, mask_row=row),
                       binding.hbsjd_adjust_logits(x, mask=mask.view(torch.uint32), mask_row=row))


def test_one_row_for_all():
    import torch
    V = 2000
    s, t = _rows(1, 1, V), _rows(2, 50, V)
    wide = s.expand(50, V)
    got, want = binding.hbsjd_distill(wide, t), binding.hbsjd_distill(wide.contiguous(), t)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for a, b in zip(binding.hbsjd_topk_logits(wide, 9), binding.hbsjd_topk_logits(s, 9)):
        assert torch.equal(a, b.expand_as(a))
    assert torch.equal(binding.hbsjd_adjust_logits(wide, logits_u=t, cfg_scale=2.0),
                       binding.hbsjd_adjust_logits(wide.contiguous(), logits_u=t, cfg_scale=2.0))
    with pytest.raises(binding.HbsjdError):
        binding.hbsjd_distill(t, t, grad=wide)


def test_no_rows_and_refused_tensors():
    import torch
    x = _rows(1, 4, 100)
    empty = x[:0]
    assert binding.hbsjd_adjust_logits(empty).shape == (0, 100)
    assert binding.hbsjd_topk_logits(empty, 5)[0].shape == (0, 5)
    assert binding.hbsjd_distill(empty, empty)[1].shape == (0, 100)
    v, i, r = binding.hbsjd_topk_logits(x, 5)
    calls = [
        lambda: binding.hbsjd_topk_logits(x.half(), 5), lambda: binding.hbsjd_topk_logits(x.t(), 3),
        lambda: binding.hbsjd_topk_logits(x[:, ::2], 3), lambda: binding.hbsjd_topk_logits(x, 101),
        lambda: binding.hbsjd_topk_logits(x[0], 3), lambda: binding.hbsjd_topk_logits(x, 5, temperature=0.0),
        lambda: binding.hbsjd_distill(x, x[:3]), lambda: binding.hbsjd_distill(x, x.cpu()),
        lambda: binding.hbsjd_distill(x, x, weight=torch.ones(3, device="cuda")),
        lambda: binding.hbsjd_distill(x, x, weight=torch.ones(4, device="cuda", dtype=torch.float64)),
        lambda: binding.hbsjd_distill(x, x, weight=torch.ones(8, device="cuda")[::2]),
        lambda: binding.hbsjd_distill(x, x, grad=x.bfloat16()),
        lambda: binding.hbsjd_distill_topk(x, v, i.long()), lambda: binding.hbsjd_distill_topk(x, v[:, :3], i),
        lambda: binding.hbsjd_distill_topk(x, v, i, None, reverse=0.5),
        lambda: binding.hbsjd_adjust_logits(x, bias=torch.ones(99, device="cuda")),
        lambda: binding.hbsjd_adjust_logits(x, mask=torch.ones(1, 3, device="cuda", dtype=torch.int32)),
        lambda: binding.hbsjd_adjust_logits(x, history=torch.ones(3, 3, device="cuda", dtype=torch.int32), presence=1.0),
        lambda: binding.hbsjd_adjust_logits(x, repetition=0.0),
        lambda: binding.hbsjd_adjust_logits(x, logits_u=x.bfloat16()),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(binding.HbsjdError) as e:
            call()
        assert e.value.code == -1, n


# ------------------------------------------------------------------ as they are used
def test_rules_then_verification():
    """Guided logits with masked tokens and penalties, verified: every committed token is one that the mask allows, and the
    probabilities are those of the adjusted logits."""
    import torch
    from tests import gpu_util as G
    case = G.verify_case(21, B=24, W=8, T=64, V=1024, branches=2, cfg_scale=3.0)
    B, W, V, T = case["B"], case["W"], case["V"], case["T"]
    d = {k: G.dev(case[k]) for k in ("logits", "q", "cursor", "seq", "delta", "qbase")}
    lc, lu = d["logits"].reshape(2, B * W, V)
    allowed = torch.rand(2, V, generator=_gen(1), device="cuda") < 0.5
    words = (allowed.view(2, -1, 32).long() << torch.arange(32, device="cuda")).sum(-1)
    mask = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()
    image = torch.arange(B * W, device="cuda") // W
    # position j of image b has seen its committed tokens and the drafts in front of it (entry 0 of a sequence is not used)
    seen = (d["cursor"][image] + torch.arange(B * W, device="cuda") % W).clamp(max=T).int()
    x = binding.hbsjd_adjust_logits(lc, lu, 3.0, mask=mask, mask_row=(image % 2).int(), history=d["seq"][:, 1:].contiguous(),
                                    history_row=image.int(), history_len=seen, repetition=1.2, presence=0.1)
    desc = G.verify_desc(case, 5, 3)
    desc.branches = 1
    p_out = torch.zeros((B, W, V), device="cuda")
    m_out = torch.zeros(B, dtype=torch.int32, device="cuda")
    before = d["cursor"].clone()
    binding.hbsjd_verify_static(torch.cuda.current_stream(), desc, x, d["q"], p_out, d["cursor"], d["seq"], d["delta"],
                                d["qbase"], m_out)
    torch.cuda.synchronize()
    for b in range(B):
        c0, c1 = int(before[b]), int(d["cursor"][b])
        n = min(W, T - c0)
        if n <= 0:
            continue
        want = torch.softmax(x.view(B, W, V)[b, :n].double(), -1)
        assert bool(((p_out[b, :n].double() - want).abs() <= 1e-6 + 1e-5 * want).all())
        assert c1 > c0
        assert bool(allowed[b % 2][d["seq"][b, c0 + 1:c1 + 1].long()].all())


def test_a_step_of_distillation_from_stored_lists():
    """Teacher's lists once, then steps on the student's head through autograd: the kernel's gradient moves the weights as the
    64-bit loss's does."""
    import torch
    torch.manual_seed(0)
    rows, D, V = 48, 64, 2000
    h = torch.randn(rows, D, device="cuda", dtype=torch.float64)
    head = torch.randn(V, D, device="cuda", dtype=torch.float64) * 0.2
    teacher = torch.randn(rows, V, device="cuda") * 2
    values, indices, rest = binding.hbsjd_topk_logits(teacher, 100)
    w = torch.full((rows,), 1.0 / rows, device="cuda")
    own = head.float().requires_grad_()
    logits = h.float() @ own.t()
    loss, grad = binding.hbsjd_distill_topk(logits.detach(), values, indices, rest, w, forward=0.5, reverse=0.5)
    logits.backward(grad)
    ref = head.clone().requires_grad_()
    x = h @ ref.t()
    y = torch.cat([values.double(), rest.double()[:, None]], 1)
    lq = torch.log_softmax(x, -1)
    others = torch.logsumexp(lq.scatter(1, indices.long(), NEG), -1, keepdim=True)
    lq = torch.cat([lq.gather(1, indices.long()), others], 1)
    lp = torch.log_softmax(y, -1)
    total = (0.5 * (lp.exp() * (lp - lq)).sum(-1) + 0.5 * (lq.exp() * (lq - lp)).sum(-1)).mean()
    total.backward()
    assert abs(float(loss.mean()) - float(total.detach())) <= 1e-4 * float(total.detach())
    # fp32 products over 64 and 48 terms of logits of size 12: 1e-5 of the largest entry and more
    assert bool(((own.grad.double() - ref.grad).abs() <= 1e-4 * ref.grad.abs().max()).all())
