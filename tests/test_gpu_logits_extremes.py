"""Divergences of rows that are masked by finite values, or come at temperatures far from one: against 64 bits."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import EXP, HALF, NEG, SUM, _compare, _distill_ref, _gen, _rows, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,rows", [(1000, 7), (16384, 6), (16384, 320), (40001, 160)])
def test_gradients_where_the_lowest_value_masks_the_student(dtype, V, rows):
    """weight * reverse / temperature^2 above 1 times the lowest value is beyond the type, and such an entry has no share: its
    gradient is -weight forward p / temperature, which is no NaN.  The lowest value on the student alone, against -1e9, against
    itself, and over a block that holds whole parts of the row."""
    import torch
    low = torch.finfo(_t(dtype)).min
    s, t = _rows(1, rows, V, 3.0, dtype), _rows(2, rows, V, 2.0, dtype)
    hide = torch.rand(rows, V, generator=_gen(3), device="cuda") < 0.3
    hide[:, 0] = False
    block = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
    block[:, V // 4:V - V // 4] = True
    kind = (torch.arange(rows, device="cuda") % 6)[:, None]
    here = torch.where(kind < 3, hide, block)
    t = torch.where(here & (kind % 3 == 1), -1e9, t.float()).to(t.dtype)
    t = torch.where(here & (kind % 3 == 2), low, t.float()).to(t.dtype)
    s = torch.where(here, low, s.float()).to(s.dtype)
    for weight, tau, a, b in ((1.0, 0.7, 0.0, 1.0), (1.0, 0.5, 0.5, 0.5), (2.0, 1.0, 0.0, 1.0), (1.0, 0.7, 0.5, 0.5), (1.0, 1.0, 0.0, 1.0),
                              (0.5, 1.0, 0.5, 0.5), (-3.0, 1.0, 0.2, 0.8), (1.0, 0.7, 1.0, 0.0), (50.0, 0.1, 0.1, 0.9)):
        w = torch.full((rows,), weight, device="cuda")
        loss, grad = binding.hbsjd_distill(s, t, w, tau, a, b)
        want, g, tl, tg = _distill_ref(s, t, w, tau, a, b)
        # The reference drops shares below 2^-126; the kernel may count those from 2^-126 / k1 on, with k1 = 2 weight reverse / tau^2 and
        # more: an entry of such a share q is off by q (a + b (|r| + KL(q || p))) weight / tau, rounded (2^-8 of it in bf16), and by
        # the sums' error of that (below 2^-8, too); no other is.  A teacher's share near 2^-126 may fall either way: a p weight / tau.
        lq, lp = torch.log_softmax(s.double() / tau, -1), torch.log_softmax(t.double() / tau, -1)
        q, r = lq.exp(), (lq - lp).abs()
        edge = (q < 1.01 * 2.0 ** -126) & (q * (2 * abs(weight) * b / tau ** 2 + 2) > 2.0 ** -126)
        more = torch.where(edge, 1.01 * q * (a + b * (r + (q * r).sum(-1, keepdim=True))) * abs(weight) / tau, 0.0)
        more = more + 1.01 * 2.0 ** -126 * a * abs(weight) / tau
        tg = tg + more
        assert bool(torch.isfinite(grad).all()), (weight, tau, a, b, torch.isnan(grad).sum(-1).unique())
        both = torch.arange(rows, device="cuda") % 3 != 0       # (the loss too, where forward KL does not pass what fp32 holds)
        if a == 0:
            both[:] = True
        _compare(loss[both], grad[both], tuple(x[both] for x in (want, g, tl, tg)), dtype)
        # on the student alone: a KL(p || q) beyond fp32's reach; the gradients stay
        if a:
            assert bool((loss[~both] > 1e30).all())
            err = (grad.double() - g).abs()
            # (the tolerance without forward KL's huge logarithms)
            p = lp.exp()
            fin = torch.where(q > 0, (s.double() - t.double()).abs() / tau, 0.0)
            size = a * (q + p) + b * q * (fin + (q * fin).sum(-1, keepdim=True) + 1)
            tol = abs(weight) / tau * size * (2 * SUM + EXP * 150) + HALF[dtype] * g.abs() + more + 1e-37
            assert bool((err <= tol)[~both].all()), float((err / tol)[~both].max())


def test_the_lowest_value_beside_logits_that_are_nearly_as_large():
    """The lowest value less a reference of 2e31 is infinite, and the entry has no share all the same."""
    import torch
    for V, rows in ((16384, 4), (16384, 320)):
        s, t = _rows(1, rows, V), _rows(2, rows, V, 2.0)
        s[:, 100], t[:, 100] = 2e31, 2e31
        s[:, 9000:9004], t[:, 9000:9004] = torch.finfo(torch.float32).min, -1e9
        w = torch.full((rows,), 2.0, device="cuda")
        loss, grad = binding.hbsjd_distill(s, t, w, 0.7, 0.5, 0.5)
        assert not bool(loss.any()) and not bool(grad.any())    # both have all mass on one token


@pytest.mark.parametrize("V,rows", [(9, 4), (1001, 320), (16385, 5)])
def test_temperatures_near_none(V, rows):
    """At a temperature far below the logits' differences both distributions are one token each, and the gradient is
    weight forward / temperature at the student's less the same at the teacher's: that of KL(q || p) is q (d - E_q d), which is none."""
    import torch
    s, t = _rows(1, rows, V), _rows(2, rows, V, 2.0)
    t[::2, 3], s[::2, 3] = 50.0, 50.0                           # (every other row: the same token)
    w = torch.full((rows,), 0.5, device="cuda")
    at = torch.arange(rows, device="cuda")
    for tau in (1e-10, 1e-20, 1e-30):
        for a, b in ((1.0, 0.0), (0.0, 1.0), (0.5, 0.5)):
            _, grad = binding.hbsjd_distill(s, t, w, tau, a, b)
            want = torch.zeros(rows, V, dtype=torch.float64, device="cuda")
            want[at, s.argmax(-1)] += 0.5 * a / tau
            want[at, t.argmax(-1)] -= 0.5 * a / tau
            # shares of 1 by ex2 and lg2, temperature and its inverse rounded, products; and d - E_q d of two that are alike, each
            # rounded by its size
            tol = (2 * SUM + 8 * HALF["fp32"]) * want.abs()
            tol[at, s.argmax(-1)] += 0.5 * b / tau * 4 * HALF["fp32"] * ((s - t).abs().amax(-1) * 2 / tau).double()
            assert bool(torch.isfinite(grad).all()) and bool(((grad.double() - want).abs() <= tol).all()), (tau, a, b)


def _list_ref(s, values, indices, rest, tau, a, b):
    """Loss, gradient and bounds of their errors over the listed tokens and the others, whose shares are taken against their own
    largest: at -1e30 64 bits keep nothing of a logarithm that is added to a logit."""
    import torch
    x = s.double()
    z = (x - x.amax(-1, keepdim=True)) / tau
    at = indices.long()
    zo = z.scatter(1, at, NEG)
    mo = zo.amax(-1, keepdim=True)
    share = torch.exp(zo - mo)
    no = share.sum(-1, keepdim=True)
    lq = torch.log_softmax(torch.cat([z.gather(1, at), mo + no.log()], 1), -1)
    lp = torch.log_softmax(torch.cat([values.double() / tau, rest.double()[:, None]], 1), -1)
    q, p, r = lq.exp(), lp.exp(), lq - lp
    F, R = (-p * r).sum(-1, keepdim=True), (q * r).sum(-1, keepdim=True) if b else 0.0
    g = a * (q - p) + (b * q * (r - R) if b else 0.0)
    # masses of sums and exponentials: each outcome's share is off by SUM and by EXP times its logarithm, which is below 90 or not there
    size = a * (q + p) + (b * q * (r.abs() + R.abs() + 1) if b else 0.0)
    full = lambda y: (y[:, -1:] * share / no).scatter(1, at, y[:, :-1])
    loss = (a * F + b * R)[:, 0]
    tl = ((a * p + b * q) * (r.abs() + 1)).sum(-1)
    return loss, full(g) / tau, (2 * SUM + 90 * EXP) * tl, (3 * SUM + 90 * EXP) * full(size) / tau


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,rows,shift", [(9, 3, 0), (1001, 300, 1), (16385, 4, 0), (16385, 300, 3)])
def test_lists_beside_others_of_one_very_low_value(dtype, V, rows, shift):
    """-1e30, which many programs mask with, on all tokens or on all that are not listed: each has the same share, whatever fills
    the row up to whole groups.  And temperatures at which such a value is not low."""
    import torch
    k = 3
    indices = torch.stack([torch.randperm(V, generator=_gen(r), device="cuda")[:k] for r in range(rows)]).int()
    values = torch.randn(rows, k, generator=_gen(1), device="cuda")
    rest = torch.randn(rows, generator=_gen(2), device="cuda")
    low = _rows(0, rows, V, 0.0, dtype, 0, shift).fill_(-1e30)
    cases = [(low, 1.0), (low, 100.0)]
    some = _rows(0, rows, V, 0.0, dtype, 0, shift).fill_(-1e30)
    some.scatter_(1, indices.long(), torch.randn(rows, k, generator=_gen(3), device="cuda").to(some.dtype))
    cases.append((some, 1.0))
    cases += [(_rows(4, rows, V, 3.0, dtype, 0, shift), tau) for tau in (1e28, 1e29, 1e30, 3e31, 1e36)]
    for s, tau in cases:
        y = values * tau if tau > 1e3 else values
        for a, b in ((1.0, 0.0), (0.5, 0.5)):
            loss, grad = binding.hbsjd_distill_topk(s, y, indices, rest, None, tau, a, b)
            want, g, tl, tg = _list_ref(s, y, indices, rest, tau, a, b)
            gone = want > 1e25                                  # (the student has nothing where the teacher's rest has)
            assert torch.equal(gone, loss > 1e25)
            assert bool(((loss.double() - want).abs() <= tl + HALF["fp32"] * want)[~gone].all()), (tau, a, b)
            if b and bool(gone.any()):
                continue                                        # (KL(q || p) takes no part in what is asked here)
            assert bool(((grad.double() - g).abs() <= tg + HALF[dtype] * g.abs() + 1e-37).all()), (tau, a, b)


@pytest.mark.parametrize("ds,dt", [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("V,rows,shift", [(9, 3, 0), (1001, 300, 1), (16385, 4, 0), (16385, 300, 3)])
def test_rows_of_one_very_low_value_and_temperatures_beyond_it(ds, dt, V, rows, shift):
    """As above, of two whole rows: uniform at -1e30 on one side or both; at temperatures from 1e28 on both rows are uniform, and the
    divergence is none, whatever the two types make of the value that fills them up."""
    import torch
    s, t = _rows(1, rows, V, 3.0, ds, 0, shift), _rows(2, rows, V, 2.0, dt, 0, shift)
    low_s, low_t = _rows(0, rows, V, 0.0, ds, 0, shift).fill_(-1e30), _rows(0, rows, V, 0.0, dt, 0, shift).fill_(-1e30)
    w = torch.ones(rows, device="cuda")
    for a, b in ((1.0, 0.0), (0.0, 1.0), (0.5, 0.5)):
        for x, y in ((low_s, t), (s, low_t), (low_s, low_t)):
            for tau in (1.0, 0.7):
                # (-1e30 / tau is uniform too, and 64 bits take its maximum off first)
                _compare(*binding.hbsjd_distill(x, y, w, tau, a, b), _distill_ref(x, y, w, tau, a, b), ds)
        for tau in (1e28, 1e29, 1e30, 3e31, 1e36):
            loss, grad = binding.hbsjd_distill(s, t, None, tau, a, b)
            # |d| / tau is below 40 / 1e28: the loss has its sums' error of that, and the gradient q - p of two equal masses
            assert float(loss.abs().max()) <= 40 / tau, (tau, a, b, float(loss.abs().max()))
            assert float(grad.abs().max()) * tau <= (3 * SUM + 20 * EXP) / V, (tau, a, b)
