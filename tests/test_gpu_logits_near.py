"""Divergences of a student that is near its teacher, where distillation ends: the loss is small beside the logarithms it is made of, and
keeps its digits.  Against 64 bits, with tolerances that shrink with the rows' distance."""
import math

import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import EXP, HALF, NEG, SUM, _gen, _rows, _t

pytestmark = pytest.mark.gpu

WEIGHTS = ((1.0, 0.0), (0.0, 1.0), (0.3, 0.9), (0.5, 0.5))
EPS = (1e-3, 3e-3, 1e-2, 3e-2, 0.1, 0.3)
ULP = HALF["fp32"]


def _near(lq, lp, V, a, b, apart, limit=1 / 64, equal=True):
    """Loss over outcomes of logarithms lq, lp, and the bound of its error.

    r = log q / p of an outcome is off by the roundings of both its logits against references (each below |log share| + log V in
    temperatures) and of their difference, ULP of those, and by what all share, which counts by its square: two sums' errors
    and those of logarithms.  An error of r moves p (e^r - 1 - r) by p |e^r - 1| of it; p is off by SUM and by EXP of its logarithm,
    which moves its term in proportion.  Terms of |r| above 3/4 are differences of p, q and p r, each good to 1e-5.  Divergences
    above the limit (`apart` times that: either way may have been taken near it), and those at equal weights if `equal`, are sums weighted by d, of which no
    reference takes more than the largest |r| off: SUM of them, and that of two sums at unequal weights."""
    import torch
    q, p = lq.exp(), lp.exp()
    r = torch.where((q > 0) & (p > 0), lq - lp, 0.0)
    F = torch.where(p > 0, -p * (lq - lp), 0.0).sum(-1) if a else torch.zeros_like(q[:, 0])
    R = torch.where(q > 0, q * (lq - lp), 0.0).sum(-1) if b else torch.zeros_like(q[:, 0])
    z = torch.where((q > 0) & (p > 0), lq.abs() + lp.abs(), 0.0) + 2 * math.log(V)
    own = ULP * (z + 4 * r.abs())
    far = torch.where(r.abs() > 0.7, (p + q) * (1 + r.abs()), 0.0).sum(-1) * 1e-5

    def tight(f, x, kl):
        return (f * torch.expm1(x).abs() * own).sum(-1) + kl * (SUM + 2e-6) + (EXP * f * z * x * x).sum(-1) + far + (2 * SUM) ** 2

    wide = SUM * ((q + p) * (r.abs() + 2 * r.abs().amax(-1, keepdim=True))).sum(-1)
    if a == b and equal:
        tol = a * wide
    else:
        near = (F < apart * limit) & (R < apart * limit)
        tol = torch.where(near, a * tight(p, r, F) + b * tight(q, -r, R), (a + b) * (wide + 2 * SUM))
    return a * F + b * R, tol


@pytest.mark.parametrize("ds,dt", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16")])
@pytest.mark.parametrize("V,rows,pad,shift", [(7, 5, 0, 0), (1000, 5, 1, 1), (1000, 700, 0, 0), (16384, 6, 0, 0), (16384, 500, 0, 0),
                                              (40001, 200, 0, 0)])
def test_rows_that_are_near(ds, dt, V, rows, pad, shift):
    import torch
    small = 0
    for n, eps in enumerate(EPS):
        s = _rows(n, rows, V, 3.0, ds, pad, shift)
        t = (s.float() + eps * torch.randn(rows, V, generator=_gen(9 + n), device="cuda")).to(_t(dt))
        t[rows - 1] = s[rows - 1].to(t.dtype)                   # (one of equal rows, as far as the types allow)
        hide = torch.rand(rows, V, generator=_gen(50 + n), device="cuda") < 0.2
        hide[:, V // 2] = False
        hide[::2] = False
        s[hide], t[hide] = NEG, NEG                             # every other row is masked on both sides
        for tau in (1.0, 2.0):
            lq, lp = torch.log_softmax(s.double() / tau, -1), torch.log_softmax(t.double() / tau, -1)
            for a, b in WEIGHTS:
                loss, _ = binding.hbsjd_distill(s, t, None, tau, a, b, want_grad=False)
                want, tol = _near(lq, lp, V, a, b, 0.99)
                assert bool(((loss.double() - want).abs() <= tol + ULP * want).all()), (eps, tau, a, b, loss, want, tol)
                assert torch.equal(binding.hbsjd_distill(s, t, None, tau, a, b)[0], loss)
                small += int((tol < 0.05 * want).sum())
    assert small > 20 * rows                                    # (the tolerance is below a twentieth of most)


def test_near_rows_that_a_mask_sets_apart_on_one_side():
    """KL(p || q) of a teacher that masks what the student hardly takes, and KL(q || p) the other way: finite and small; the other
    direction is infinite and has no weight."""
    import torch
    for V, rows in ((1000, 40), (16384, 6), (16384, 300)):
        s = _rows(1, rows, V)
        t = s + 0.003 * torch.randn(rows, V, generator=_gen(2), device="cuda")
        low = s < s.amax(-1, keepdim=True) - 16
        low[:, 0] = False
        masked = t.masked_fill(low, NEG)
        lq, lp = torch.log_softmax(s.double(), -1), torch.log_softmax(masked.double(), -1)
        for w in (1.0, 0.7):
            loss, _ = binding.hbsjd_distill(s, masked, None, 1.0, w, 0.0)
            want, tol = _near(lq, lp, V, w, 0.0, 0.99)
            tol = tol + SUM * torch.where(low, lq.exp(), 0.0).sum(-1)
            assert bool(low.any()) and bool(((loss.double() - want).abs() <= tol).all())
            loss, _ = binding.hbsjd_distill(masked, s, None, 1.0, 0.0, w)
            want, tol = _near(lp, lq, V, 0.0, w, 0.99)
            tol = tol + SUM * torch.where(low, lq.exp(), 0.0).sum(-1)
            assert bool(((loss.double() - want).abs() <= tol).all())


def test_near_rows_among_others_and_rows_left_out():
    """Rows of every distance after one another in the same CTAs, some left out: each as it is alone."""
    import torch
    for V, rows in ((700, 3000), (30000, 400)):
        s = _rows(1, rows, V)
        eps = torch.tensor(EPS + (3.0,), device="cuda")[torch.randint(0, 7, (rows,), generator=_gen(3), device="cuda")]
        t = s + eps[:, None] * torch.randn(rows, V, generator=_gen(2), device="cuda")
        w = (torch.rand(rows, generator=_gen(4), device="cuda") < 0.7).float()
        every = torch.ones_like(w)
        one = binding.hbsjd_distill(s, t, every, 1.0, 1.0, 0.0)
        loss, grad = binding.hbsjd_distill(s, t, w, 1.0, 1.0, 0.0)
        assert torch.equal(loss, torch.where(w == 0, 0.0, one[0])) and torch.equal(grad, torch.where(w[:, None] == 0, 0.0, one[1]))
        want, tol = _near(torch.log_softmax(s.double(), -1), torch.log_softmax(t.double(), -1), V, 1.0, 0.0, 0.99)
        assert bool(((one[0].double() - want).abs() <= tol + ULP * want).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,k,rows,pad,shift", [(9, 4, 5, 0, 0), (1000, 1, 5, 1, 1), (1000, 64, 700, 0, 0), (16384, 64, 6, 0, 0), (16384, 64, 500, 0, 0),
                                                (16384, 1024, 8, 0, 0), (40001, 200, 200, 0, 0)])
def test_lists_of_a_near_teacher(dtype, V, k, rows, pad, shift):
    """The same over the listed tokens and all others as one.  What all listed tokens share of an error, and what the others have of one,
    count by the square and by the difference of the listed masses: each is two sums' errors and the roundings of ten logarithms no
    larger than the logits, the rest and log V = 11 in temperatures."""
    import torch
    small = 0
    for n, eps in enumerate(EPS):
        s = _rows(n, rows, V, 3.0, dtype, pad, shift)
        t = s.float() + eps * torch.randn(rows, V, generator=_gen(9 + n), device="cuda")
        t[rows - 1] = s[rows - 1].float()
        for tau in (1.0, 2.0):
            values, indices, rest = binding.hbsjd_topk_logits(t, k, tau)
            x, at = s.double() / tau, indices.long()
            lq = torch.log_softmax(torch.cat([x.gather(1, at), torch.logsumexp(x.scatter(1, at, NEG), -1, keepdim=True)], 1), -1)
            lp = torch.log_softmax(torch.cat([values.double() / tau, rest.double()[:, None]], 1), -1)
            dr = 2 * SUM + 10 * ULP * (torch.maximum(x.abs().amax(-1), t.double().abs().amax(-1) / tau) + 22)
            apart = (lq[:, -1].exp() - lp[:, -1].exp()).abs()
            for a, b in WEIGHTS:
                loss, _ = binding.hbsjd_distill_topk(s, values, indices, rest, None, tau, a, b, want_grad=False)
                want, tol = _near(lq, lp, V, a, b, 0.99, 1 / 16, False)
                tol = tol + (a + b) * (apart * dr + torch.where(want > 0.9 * min(a + b, 1) / 16, dr, 0.0))
                assert bool(((loss.double() - want).abs() <= tol + ULP * want).all()), (eps, tau, a, b, loss, want, tol)
                assert torch.equal(binding.hbsjd_distill_topk(s, values, indices, rest, None, tau, a, b)[0], loss)
                small += int((tol < 0.1 * want).sum())
    assert small > 12 * rows


def test_near_lists_among_others_and_rows_left_out():
    import torch
    for V, k, rows in ((700, 20, 3000), (60000, 50, 400)):
        s = _rows(1, rows, V)
        eps = torch.tensor(EPS + (3.0,), device="cuda")[torch.randint(0, 7, (rows,), generator=_gen(3), device="cuda")]
        lists = binding.hbsjd_topk_logits(s + eps[:, None] * torch.randn(rows, V, generator=_gen(2), device="cuda"), k)
        w = (torch.rand(rows, generator=_gen(4), device="cuda") < 0.7).float()
        one = binding.hbsjd_distill_topk(s, *lists, torch.ones_like(w), 1.0, 0.5, 0.5)
        loss, grad = binding.hbsjd_distill_topk(s, *lists, w, 1.0, 0.5, 0.5)
        assert torch.equal(loss, torch.where(w == 0, 0.0, one[0])) and torch.equal(grad, torch.where(w[:, None] == 0, 0.0, one[1]))
        assert bool((one[0] >= 0).all())
