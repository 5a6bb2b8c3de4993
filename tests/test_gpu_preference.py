"""hbsjd_preference_loss against its definition in 64 bits."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _gen, _rows
from tests.token_reference import HALF, NEG, STEP, Rows, near, sampled

pytestmark = pytest.mark.gpu

KINDS = [("sigmoid", 0.1, 0.0, 0.0), ("sigmoid", 1.0, 0.2, 0.5), ("sigmoid", 0.3, 1.0, -0.3), ("hinge", 0.5, 0.0, 0.25), ("square", 0.2, 0.0, 0.0)]


def _loss(h, kind, beta, smoothing, margin):
    import torch
    if kind == "square":
        return (h - 1 / (2 * beta)) ** 2
    z = beta * h - margin
    if kind == "hinge":
        return (1 - z).clamp(min=0)
    F = torch.nn.functional.logsigmoid
    return -(1 - smoothing) * F(z) - smoothing * F(-z)


def _check(x, t, lengths, dtype, ref=None, w=None, pw=None, tau=1.0, kind="sigmoid", beta=0.1, smoothing=0.0, margin=0.0,
           interleaved=False, front=0, grad=None):
    import torch
    rows, P = x.shape[0], len(lengths) // 2
    ends = torch.tensor([front] + lengths).cumsum(0)
    offsets = ends.int().cuda()
    r = Rows(x, t, tau)
    got = binding.hbsjd_preference_loss(x, t, offsets, ref, w, pw, tau, beta, kind, smoothing, margin, interleaved, grad=grad)
    loss, g, sums = got
    l = torch.where(r.live, r.l, 0.0)
    wd = torch.ones_like(l) if w is None else w.double()
    refd = torch.zeros_like(l) if ref is None else ref.double()
    use = (wd != 0)
    terms = torch.where(use, wd * (l - refd), 0.0)
    off = torch.where(use, wd.abs() * (r.dl * r.live + STEP * l.abs()), 0.0)
    S = torch.stack([terms[ends[i]:ends[i + 1]].sum() for i in range(2 * P)])
    dS = torch.stack([off[ends[i]:ends[i + 1]].sum() for i in range(2 * P)])
    near(sums, S, dS, HALF["fp32"])
    ci = [2 * p if interleaved else p for p in range(P)]
    ri = [2 * p + 1 if interleaved else P + p for p in range(P)]
    h = (S[ci] - S[ri]).requires_grad_()
    dh = (dS[ci] + dS[ri]).detach()
    want = _loss(h, kind, beta, smoothing, margin)
    per, = torch.autograd.grad(want.sum(), h)
    # slopes a little to either side: how far h's own error takes loss and slope (losses are convex)
    around = []
    for s in (-1, 1):
        hs = (h.detach() + s * dh).requires_grad_()
        around.append(torch.autograd.grad(_loss(hs, kind, beta, smoothing, margin).sum(), hs)[0])
    steep = torch.maximum(around[0].abs(), around[1].abs())
    near(loss, want.detach(), steep * dh + 1e-37, 2 * HALF["fp32"])
    pair_w = torch.ones(P, device="cuda").double() if pw is None else pw.double()
    a, da = torch.zeros_like(l), torch.zeros_like(l)
    for p in range(P):
        for i, sign in ((ci[p], 1.0), (ri[p], -1.0)):
            at = slice(int(ends[i]), int(ends[i + 1]))
            a[at] = sign * per[p] * pair_w[p] * wd[at]
            da[at] = ((around[1] - around[0]).abs()[p] + 4 * STEP * per[p].abs()) * pair_w[p].abs() * wd[at].abs()
    wg, bg = r.gradient(a, None, torch.ones_like(a), da)
    near(g, wg, bg, HALF[dtype])
    # less asked for: the same bits
    again = binding.hbsjd_preference_loss(x, t, offsets, ref, w, pw, tau, beta, kind, smoothing, margin, interleaved, want_grad=False)
    if grad is None:
        assert torch.equal(again[0], loss) and torch.equal(again[2], sums) and again[1] is None
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(2, 0, 0), (33, 0, 1), (1000, 3, 0), (4099, 0, 0), (16384, 0, 0), (20011, 0, 3), (65537, 1, 0)])
def test_losses_and_gradients(V, pad, shift, dtype):
    import torch
    lengths, g = [5, 1, 9, 0, 7, 12], _gen(V)
    rows = sum(lengths) + 4                      # two rows in front of all sequences, two behind
    x = _rows(V, rows, V, 3.0, dtype, pad, shift)
    t = sampled(x, 1.0, g)
    t[4], t[9] = -1, V
    ref = (Rows(x, t, 1.0).l + torch.randn(rows, generator=g, device="cuda") * 0.5).float()
    ref[4] = ref[9] = 0.0
    w = torch.rand(rows, generator=g, device="cuda")
    w[::6] = 0.0
    pw = torch.rand(3, generator=g, device="cuda")
    for i, (kind, beta, s, m) in enumerate(KINDS):
        _check(x, t, lengths, dtype, ref, w, pw, 1.0, kind, beta, s, m, interleaved=i % 2 == 0, front=2)
    _check(x, t, lengths, dtype, None, w / 8, None, 0.9, interleaved=True, front=0)
    _check(x, t, lengths, dtype, ref, None, pw, 1.0, front=4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pairs,longest,V", [(1, 1, 4096), (1, 700, 1000), (3, 300, 4099), (40, 33, 2500), (2, 130, 16384), (7, 60, 20011), (300, 2, 300)])
def test_pairs_and_lengths(pairs, longest, V, dtype):
    import torch
    g = _gen(longest)
    lengths = [1 + int(v) for v in torch.randint(0, longest, (2 * pairs,), generator=torch.Generator().manual_seed(pairs))]
    rows = sum(lengths)
    x = _rows(V, rows, V, 3.0, dtype)
    t = sampled(x, 1.0, g)
    ref = (Rows(x, t, 1.0).l + torch.randn(rows, generator=g, device="cuda") * 0.2).float()
    for interleaved in (False, True):
        got = _check(x, t, lengths, dtype, ref, interleaved=interleaved, beta=0.3)
        offsets = torch.tensor([0] + lengths).cumsum(0).int().cuda()
        for _ in range(3):                       # the same bits every time
            again = binding.hbsjd_preference_loss(x, t, offsets, ref, beta=0.3, interleaved=interleaved)
            assert all(torch.equal(u, v) for u, v in zip(got, again))


def test_gradient_in_place_of_the_logits():
    import torch
    x = _rows(1, 60, 3000)
    t, offsets = sampled(x, 1.0, _gen(1)), torch.tensor([0, 10, 20, 45, 60], device="cuda").int()
    want = binding.hbsjd_preference_loss(x, t, offsets)
    got = binding.hbsjd_preference_loss(x, t, offsets, grad=x)
    assert got[1] is x and all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_without_mass_and_without_end():
    import torch
    x = _rows(1, 12, 500)
    t, offsets = torch.arange(12, device="cuda").int(), torch.tensor([0, 3, 6, 9, 12], device="cuda").int()
    x[1], x[4, 4], x[7, 3] = NEG, NEG, float("nan")
    # pairs (0..2, 6..8): one row without mass, one NaN; (3..5, 9..11): a token without mass
    loss, g, sums = binding.hbsjd_preference_loss(x, t, offsets)
    assert sums[0] == NEG and sums[1] == NEG and bool(torch.isnan(sums[2])) and bool(torch.isfinite(sums[3]))
    assert bool(torch.isnan(loss[0])) and loss[1] == float("inf")
    # far apart: the loss is h itself, and the slope one of its ends
    y = _rows(2, 4, 100) * 50
    t2 = torch.stack([y[0].argmax(), y[1].argmax(), y[2].argmin(), y[3].argmin()]).int()
    o2 = torch.tensor([0, 2, 4], device="cuda").int()
    for swap in (False, True):
        order = [2, 3, 0, 1] if swap else [0, 1, 2, 3]
        _check(y[order].contiguous(), t2[order].contiguous(), [2, 2], "fp32", beta=5.0)


def test_offsets_that_make_no_sense():
    """Nothing is read or written out of range, and everything says so."""
    import torch
    x = _rows(1, 20, 300)
    t = torch.zeros(20, dtype=torch.int32, device="cuda")
    for bad in ([0, 5, 3], [0, 5, 21], [-1, 5, 10], [0, 2 ** 31 - 1, 10], [5, 4, 3], [0, -2 ** 31, 20]):
        loss, g, sums = binding.hbsjd_preference_loss(x, t, torch.tensor(bad, device="cuda").int())
        assert bool(torch.isnan(loss).all()) and bool(torch.isnan(sums).all()) and bool(torch.isnan(g).all())


def test_captured_replayed_and_beside_itself():
    import torch
    x, t = _rows(1, 200, 5000), torch.randint(0, 5000, (200,), device="cuda").int()
    offsets = torch.tensor([0, 60, 90, 150, 200], device="cuda").int()
    want = binding.hbsjd_preference_loss(x, t, offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = binding.hbsjd_preference_loss(x, t, offsets)
    sides = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        graph.replay()
        # other calls at the same time, each with its own workspace
        more = []
        for s in sides:
            s.wait_stream(torch.cuda.current_stream())
            more.append(binding.hbsjd_preference_loss(x, t, offsets, stream=s))
        for s in sides:
            torch.cuda.current_stream().wait_stream(s)
        for m in (got, *more):
            assert all(torch.equal(a, b) for a, b in zip(m, want))
    x.copy_(_rows(3, 200, 5000))
    offsets.copy_(torch.tensor([0, 10, 20, 30, 200]))
    graph.replay()
    want = binding.hbsjd_preference_loss(x, t, offsets)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals_of_tensors():
    import torch
    x, t = _rows(1, 8, 50), torch.zeros(8, dtype=torch.int32, device="cuda")
    o = torch.tensor([0, 4, 8], device="cuda").int()
    for call in (lambda: binding.hbsjd_preference_loss(x, t, o.long()), lambda: binding.hbsjd_preference_loss(x, t, o[:2]),
                 lambda: binding.hbsjd_preference_loss(x, t, torch.cat([o, o[2:]])), lambda: binding.hbsjd_preference_loss(x, t, None),
                 lambda: binding.hbsjd_preference_loss(x, t, o, kind="none"), lambda: binding.hbsjd_preference_loss(x, t, o, beta=0.0),
                 lambda: binding.hbsjd_preference_loss(x, t, o, smoothing=1.5), lambda: binding.hbsjd_preference_loss(x, t, o, kind="hinge", smoothing=0.1),
                 lambda: binding.hbsjd_preference_loss(x, t, o, kind="square", margin=0.1), lambda: binding.hbsjd_preference_loss(x, t, o, x[:, 0]),
                 lambda: binding.hbsjd_preference_loss(x, t, o, pair_weight=torch.ones(2, device="cuda")),
                 lambda: binding.hbsjd_preference_loss(x[:0], t[:0], o)):
        with pytest.raises(binding.HbsjdError) as e:
            call()
        assert e.value.code == -1


def test_more_pairs_than_ctas():
    """Thousands of pairs of a position or two, some empty."""
    import torch
    g = torch.Generator().manual_seed(5)
    lengths = [int(v) for v in torch.randint(0, 4, (2 * 3001,), generator=g)]
    rows = sum(lengths)
    x = _rows(3, rows, 64)
    t = sampled(x, 1.0, _gen(3))
    ref = Rows(x, t, 1.0).l.float() + 0.3
    for interleaved in (False, True):
        _check(x, t, lengths, "fp32", ref, interleaved=interleaved, beta=0.5)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(16384, 1, 0), (4099, 2, 1), (20000, 1, 3), (513, 3, 2)])
def test_gradients_that_lie_otherwise_than_the_logits(V, pad, shift, dtype):
    import torch
    lengths = [200, 30, 77, 100]
    x = _rows(V, 407, V, 3.0, dtype, pad, shift)
    t = sampled(x, 1.0, _gen(1))
    _check(x, t, lengths, dtype, beta=0.02)
    grad = torch.empty(407, V + 5, device="cuda", dtype=x.dtype)[:, 3:V + 3]
    _check(x, t, lengths, dtype, beta=0.02, grad=grad)


@pytest.mark.parametrize("rows,V", [(40, 3000), (400, 3000), (200, 20011)])
def test_nan_slopes_reach_every_entry(rows, V):
    """Offsets that make no sense, and a NaN reference: entries without any share are NaN, too."""
    import torch
    x = _rows(1, rows, V) * 40
    x[:, ::7] = NEG
    for dtype in (torch.float32, torch.bfloat16):
        y = x.to(dtype)
        t = torch.ones(rows, dtype=torch.int32, device="cuda")
        for pad in (0, 1):
            grad = torch.empty(rows, V + pad, device="cuda", dtype=dtype)[:, :V]
            g = binding.hbsjd_preference_loss(y, t, torch.tensor([0, 9, 3], device="cuda").int(), grad=grad)[1]
            assert bool(torch.isnan(g).all())
            ref = torch.zeros(rows, device="cuda")
            ref[3] = float("nan")
            half = torch.tensor([0, 10, 20, 30, 40], device="cuda").int()
            loss, g, _ = binding.hbsjd_preference_loss(y, t, half, ref, interleaved=True, grad=grad)
            assert bool(torch.isnan(loss[0])) and bool(torch.isfinite(loss[1]))
            assert bool(torch.isnan(g[:20]).all()) and bool(torch.isfinite(g[20:]).all())
