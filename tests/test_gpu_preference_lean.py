"""What all rows' log-probabilities are off alike in hbsjd_preference_loss: it adds up over a sequence, and does not cancel between sequences of
different lengths.  Read from the sums of sequences of one row, against references that are the log-probabilities themselves in
fp32, so that a sum is what l's own rounding leaves (1e-6 at most, itself rounded to 1e-13)."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _gen, _rows
from tests.token_reference import STEP, Rows, sampled

pytestmark = pytest.mark.gpu


def _off(x, t, l, tau):
    """Errors of every row's log-probability, l in 64 bits."""
    import torch
    rows = x.shape[0]
    ref = l.float()
    offsets = torch.arange(rows + 1, device="cuda").int()
    _, _, sums = binding.hbsjd_preference_loss(x, t, offsets, ref, temperature=tau, want_grad=False)
    return sums.double() - (l - ref.double())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows", [40, 400])
@pytest.mark.parametrize("V", [257, 1025, 4097, 16385, 65537])
def test_rows_of_one_value(V, rows, dtype):
    """All others are alike, 2^k of them: every exponential is 1, their sum is exact, and so is its logarithm but for k ln2's two floats.
    What is left: log(1 + 2^-k) < 2^-8 with four half steps and 1e-8 of itself, and the rounding of what is added to it: less than
    2^-8 (5 2^-24 + 1e-8) < 1.3e-9; with as much for the last sum's own rounding below 3e-9."""
    import torch
    x = torch.full((rows, V), 1.25, device="cuda").to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    t = torch.randint(0, V, (rows,), generator=_gen(V), device="cuda").int()
    l = torch.full((rows,), -float(torch.tensor(V).double().log()), device="cuda", dtype=torch.float64)
    for tau in (1.0, 0.7):
        assert float(_off(x, t, l, tau).abs().max()) < 3e-9


@pytest.mark.parametrize("V,scale,tau", [(V, s, tau) for V in (2, 33, 1000, 16384, 131072) for s, tau in ((0.1, 1.0), (3.0, 1.0), (3.0, 0.7), (10.0, 1.0))])
def test_mean_over_rows(V, scale, tau):
    """Of one sign are an exponential's 2^-22 and what c = log2(e) / tau is off by, three half steps of its exponents; roundings are of either sign, so
    that their mean is within six deviations of none."""
    import torch
    rows = 1024
    x = _rows(V, rows, V, scale)
    t = sampled(x, tau, _gen(V))
    off, lean = [], []
    for at in range(0, rows, 256):
        s = slice(at, at + 256)
        r = Rows(x[s], t[s], tau)
        others = r.q.scatter(1, r.t[:, None], 0.0)
        far = (others * r.z.abs()).sum(-1)
        off.append(_off(x[s], t[s], r.l, tau))
        lean.append(r.qo * 2.0 ** -22 + 3 * STEP * far)
    off, lean = torch.cat(off), torch.cat(lean)
    assert float(off.mean().abs()) <= float(lean.mean() + 6 * off.std() / rows ** 0.5)
