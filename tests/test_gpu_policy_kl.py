"""The KL term of hbsjd_policy_loss and its slope alone, against 64 bits: the references are set from the log-probabilities that the kernel itself gives, so
that their error hides none of the term's."""
import math

import pytest

from paper_2608_18183_b200 import binding
from tests.token_reference import STEP

pytestmark = pytest.mark.gpu


def _distances():
    """Multiples of 2^-20: either sign, from next to none to 16, and just inside and outside of where a formula may change."""
    import torch
    n = torch.arange(-400, 401).double()
    wide = torch.sign(n) * 2.0 ** (n.abs() / 17 - 19.5)
    borders = torch.tensor([b + k * 2.0 ** -20 for b in (0.25, 0.5, math.log(2), 0.75, 1.0, 2.0) for k in range(-40, 41)]).double()
    fine = torch.linspace(-1.25, 1.25, 2001).double()
    d = torch.cat([wide, borders, -borders, fine, torch.linspace(-16, 5, 1001).double()])
    return (d * 2.0 ** 20).round().div(2.0 ** 20).cuda()


@pytest.mark.parametrize("V", [2, 9001])
def test_value(V):
    """Within 8 half steps of itself.  l is a multiple of 2^-24 (V = 2), or of 2^-20: the kernel's difference of two fp32 numbers is
    rounded once, by half a step of d at most, which is (e^d - 1) / (e^d - 1 - d) times as much of the term."""
    import torch
    d = _distances()
    rows = d.numel()
    x, t = torch.zeros(rows, V, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    none = torch.zeros(rows, device="cuda")
    l = binding.hbsjd_policy_loss(x, t, none)[2]
    ref = (l.double() + d).float()
    d = ref.double() - l.double()
    for want_grad in (True, False):
        loss, _, again, _ = binding.hbsjd_policy_loss(x, t, none, ref_logp=ref, kl=1.0, want_grad=want_grad)
        assert torch.equal(again, l)
        # (e^d - 1 - d in 64 bits: by series where the difference would lose digits)
        series = d * d * (0.5 + d * (1 / 6 + d * (1 / 24 + d * (1 / 120 + d * (1 / 720 + d / 5040)))))
        want = torch.where(d.abs() < 1e-2, series, torch.expm1(d) - d)
        bound = 8 * STEP * want + STEP * d.abs() * torch.expm1(d).abs()
        assert bool(((loss.double() - want).abs() <= bound + 1e-37).all())


def test_slope():
    """e^d - 1 within five half steps of itself: the two products, and expm1f's step or the series' sum (8 of the term, 1 of the sum).  Read
    from the token's entry of rows whose other token has the same logit, over that of a slope of one."""
    import torch
    d = _distances()
    rows = d.numel()
    x, t = torch.zeros(rows, 2, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    none = torch.zeros(rows, device="cuda")
    _, one, l, _ = binding.hbsjd_policy_loss(x, t, none + 1)
    ref = (l.double() + d).float()
    d = ref.double() - l.double()
    g = binding.hbsjd_policy_loss(x, t, none, ref_logp=ref, kl=1.0)[1]
    got, want = (g[:, 0].double() / one[:, 0].double()), torch.expm1(d)
    bound = 5 * STEP * want.abs() + STEP * d.abs() * d.exp()
    assert bool(((got - want).abs() <= bound + 1e-37).all())


def test_ends():
    import torch
    x, t = torch.zeros(6, 50, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    none, inf, nan = torch.zeros(6, device="cuda"), float("inf"), float("nan")
    l = binding.hbsjd_token_logprobs(x, t)[0]
    ref = l + torch.tensor([0.0, -inf, inf, nan, 60.0, -200.0], device="cuda")
    loss, g, _, _ = binding.hbsjd_policy_loss(x, t, none, ref_logp=ref, kl=0.5)
    assert loss[0] == 0 and not bool(g[0].any())
    assert loss[1] == inf and bool(torch.isfinite(g[1]).all())
    assert loss[2] == inf and bool(torch.isnan(loss[3])) and bool(torch.isnan(g[3]).all())
    d = (ref - l).double()
    torch.testing.assert_close(loss[4:].double(), 0.5 * (torch.expm1(d) - d)[4:], rtol=8 * STEP, atol=0)
    torch.testing.assert_close(g[5], g[1], rtol=0, atol=0)
