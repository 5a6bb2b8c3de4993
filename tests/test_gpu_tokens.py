"""hbsjd_token_logprobs, hbsjd_token_logprobs_grad and hbsjd_policy_loss against their definitions in 64 bits (see token_reference.py for
the bounds)."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _gen, _rows
from tests.token_reference import HALF, NEG, Rows, away, near, policy, sampled

pytestmark = pytest.mark.gpu

SHAPES = [(1, 0, 0), (2, 0, 0), (5, 0, 1), (33, 0, 1), (1000, 3, 0), (4099, 0, 0), (8192, 0, 0), (16384, 0, 0), (20011, 0, 3),
          (8200, 8, 8), (65537, 1, 0), (131072, 0, 0)]


def _check_logprobs(x, t, tau, dtype, seed=0):
    import torch
    rows = x.shape[0]
    r = Rows(x, t, tau)
    logp, H = binding.hbsjd_token_logprobs(x, t, tau)
    live = r.live
    near(logp, torch.where(live, r.l, 0.0), torch.where(live, r.dl, 0.0), HALF["fp32"])
    near(H, torch.where(live & ~r.empty, r.H, 0.0), r.dH, HALF["fp32"])
    alone, none = binding.hbsjd_token_logprobs(x, t, tau, want_entropy=False)
    near(alone, torch.where(live, r.l, 0.0), torch.where(live, r.dl, 0.0), HALF["fp32"])
    assert none is None
    a, b = torch.randn(rows, generator=_gen(seed + 1), device="cuda"), torch.randn(rows, generator=_gen(seed + 2), device="cuda")
    for ent in (None, b):
        g = binding.hbsjd_token_logprobs_grad(x, t, a, ent, tau)
        assert g.dtype == x.dtype and g.shape == x.shape
        want, bound = r.gradient(a.double(), None if ent is None else ent.double(), torch.ones_like(r.l))
        near(g, want, bound, HALF[dtype])
    return g


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", SHAPES)
def test_logprobs_and_their_backward(V, pad, shift, dtype):
    import torch
    x = _rows(V, 9, V, 3.0, dtype, pad, shift)
    t = sampled(x, 1.3, _gen(V))
    t[3], t[4] = 0, V - 1
    t[5], t[6] = -1, V
    g = _check_logprobs(x, t, 1.3, dtype, V)
    assert not bool(g[5:7].any())
    # in place
    y = x.clone() if pad == 0 else x
    a = torch.randn(9, generator=_gen(V + 1), device="cuda")
    want = binding.hbsjd_token_logprobs_grad(y, t, a, None, 1.3)
    assert binding.hbsjd_token_logprobs_grad(y, t, a, None, 1.3, grad=y) is y
    assert torch.equal(y, want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,V,pad", [(700, 1000, 0), (3000, 4096, 0), (900, 16384, 0), (700, 20011, 0), (2500, 2501, 0), (260, 65536, 1)])
def test_many_rows_a_cta(rows, V, pad, dtype):
    """More rows than CTAs, at strides that change the rows' places behind 16 bytes, so that rows are fetched ahead in every way."""
    x = _rows(rows, rows, V, 3.0, dtype, pad, 1)
    t = sampled(x, 1.0, _gen(1))
    t[::17] = -1
    _check_logprobs(x, t, 1.0, dtype)


def test_rows_out_of_the_ordinary():
    import torch
    V = 3001
    base = _rows(1, 24, V)
    big, low = torch.finfo(torch.float32).max, torch.finfo(torch.float32).min
    x, t = base.clone(), torch.full((24,), 7, dtype=torch.int32, device="cuda")
    x[0], x[1] = NEG, NEG                       # nothing has mass; the token alone has
    x[1, 7] = 0.3
    x[2, 7] = NEG                               # the token has none
    x[3, ::2] = NEG                             # half masked, the token too or not
    x[4, 1::2] = NEG
    x[5], x[6] = low, low                       # the type's lowest value: all alike; as a mask
    x[6, 100:] = base[6, 100:]
    x[7, 5] = big
    x[8, 7] = big                               # the token has all the mass
    x[9, 7] = 30.0                              # nearly all
    x[10, 7] = 17.0
    x[11, 2000], x[11, 7] = 40.0, -40.0
    x[12] += 1000.0
    x[13] -= 1e6
    x[14] = torch.linspace(-100, 100, V, device="cuda")
    x[15] = x[14].flip(0)
    x[16, 7] = NEG
    x[16, :2900] = NEG                          # warps without an entry of mass
    x[17, :600] = x[17, :600] * 0 - 500         # a sample far below the rest
    x[18] = 0
    for tau in (1.0, 0.3, 4.0):
        _check_logprobs(x[:19], t[:19], tau, "fp32")
    y = x[:19].bfloat16()
    _check_logprobs(y, t[:19], 1.0, "bf16")


def test_nan_and_infinity_spoil_their_row_alone():
    import torch
    x, t = _rows(1, 8, 5000), torch.full((8,), 9, dtype=torch.int32, device="cuda")
    x[1, 77], x[2, 9], x[3, 4999], x[4, 9] = float("nan"), float("nan"), float("inf"), float("inf")
    good = torch.tensor([0, 5, 6, 7], device="cuda")
    one = torch.ones(8, device="cuda")
    logp, H = binding.hbsjd_token_logprobs(x, t)
    g = binding.hbsjd_token_logprobs_grad(x, t, one, one)
    loss, pg, lp, pH = binding.hbsjd_policy_loss(x, t, one, entropy=0.1, want_entropy=True)
    clean = binding.hbsjd_token_logprobs(x[good], t[good])
    for v, w in ((logp, clean[0]), (H, clean[1])):
        assert bool(torch.isnan(v[1:5]).all()) and torch.equal(v[good], w)
    for v in (loss, lp, pH):
        assert bool(torch.isnan(v[1:5]).all()) and bool(torch.isfinite(v[good]).all())
    for v in (g, pg):
        assert bool(torch.isnan(v[1:5]).all()) and bool(torch.isfinite(v[good]).all())


@pytest.mark.parametrize("tau", [4.4e-39, 1e-30, 1e-6, 1e6, 1e30, 3e38])
def test_temperatures_near_none_and_without_end(tau):
    import torch
    x, t = _rows(1, 6, 300), torch.tensor([0, 1, 2, 3, 4, 5], device="cuda").int()
    t[:3] = x[:3].argmax(-1).int()
    one = torch.ones(6, device="cuda")
    logp, H = binding.hbsjd_token_logprobs(x, t, tau)
    g = binding.hbsjd_token_logprobs_grad(x, t, one * min(1.0, tau), one * min(1.0, tau) * 0.5, tau)
    for v in (logp, H, g):
        assert not bool(torch.isnan(v).any())
    r = Rows(x, t, tau)
    if tau < 1:
        assert bool((logp[:3].double() - r.l[:3] >= -1e-5).all()) and bool((H < 1e-3).all())
    else:
        near(logp, r.l, r.dl, HALF["fp32"])
        near(H, r.H, r.dH, HALF["fp32"])


POLICY = [dict(), dict(kl=0.1), dict(bonus=0.02), dict(dual=1.5, kl=0.05, bonus=-0.01), dict(low=0.0, high=0.0), dict(low=1.0, high=5.0, dual=3.0)]


def _check_policy(x, t, A, old, ref, w, tau, dtype, low=0.2, high=0.2, dual=0.0, kl=0.0, bonus=0.0):
    import torch
    r = Rows(x, t, tau)
    how = dict(temperature=tau, clip_low=low, clip_high=high, dual_clip=dual, kl=kl, entropy=bonus)
    loss, g, logp, H = binding.hbsjd_policy_loss(x, t, A, old, ref if kl else None, w, want_entropy=True, **how)
    want, bound, slope, dslope = policy(r, A, old, ref, w, low, high, dual, kl, bonus)
    near(loss, want, bound, HALF["fp32"])
    left = ~r.live | (torch.zeros_like(r.live) if w is None else w == 0)
    near(logp, torch.where(left, 0.0, r.l), r.dl, HALF["fp32"])
    near(H, torch.where(left | r.empty, 0.0, r.H), r.dH, HALF["fp32"])
    weight = torch.ones_like(r.l) if w is None else w.double()
    b = torch.full_like(r.l, -bonus) if bonus else None
    wg, bg = r.gradient(slope, b, weight, dslope)
    near(g, wg, bg, HALF[dtype])
    # less asked for: the same bits
    loss2, none, logp2, _ = binding.hbsjd_policy_loss(x, t, A, old, ref if kl else None, w, want_grad=False, want_entropy=True, **how)
    assert none is None and torch.equal(loss, loss2) and torch.equal(logp, logp2)
    return loss, g


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,shift", [(2, 0, 0), (33, 0, 1), (1000, 3, 0), (4099, 0, 0), (16384, 0, 0), (20011, 0, 3), (65537, 1, 0)])
def test_policy_loss_and_gradient(V, pad, shift, dtype):
    import torch
    rows, g = 40, _gen(V)
    x = _rows(V, rows, V, 3.0, dtype, pad, shift)
    t = sampled(x, 0.9, g)
    t[5], t[6] = -1, V + 3
    r = Rows(x, t, 0.9)
    A = torch.randn(rows, generator=g, device="cuda")
    A[7] = 0.0
    ref = (r.l + torch.randn(rows, generator=g, device="cuda") * 0.5).float()
    ref[8] = r.l[8].float()
    w = torch.rand(rows, generator=g, device="cuda") / rows
    w[9:12] = 0.0
    for how in POLICY:
        low, high = how.get("low", 0.2), how.get("high", 0.2)
        gap = away(torch.randn(rows, generator=g, device="cuda").double() * 0.4, low, high)
        gap = torch.where(gap.abs() < 1e-3, 2e-3, gap) if low == 0 else gap
        if how.get("dual"):
            gap = torch.where((gap.exp() - how["dual"]).abs() < 1e-2, gap + 0.1, gap)
        old = (r.l - gap).float()
        _check_policy(x, t, A, old, ref, w, 0.9, dtype, **how)
    for how in POLICY[:4]:
        _check_policy(x, t, A, None, ref, None, 0.9, dtype, **how)


def test_policy_many_rows():
    import torch
    x, g = _rows(1, 2500, 5000, 3.0, "fp32"), _gen(2)
    t = sampled(x, 1.0, g)
    r = Rows(x, t, 1.0)
    A, w = torch.randn(2500, generator=g, device="cuda"), torch.ones(2500, device="cuda") / 2500
    w[::5] = 0.0
    w[1000:1700] = 0.0
    old = (r.l - away(torch.randn(2500, generator=g, device="cuda").double() * 0.2, 0.2, 0.2)).float()
    _check_policy(x, t, A, old, r.l.float() + 0.1, w, 1.0, "fp32", kl=0.04, bonus=0.01)


def test_policy_at_its_edges():
    """Ratios without end and of zero, advantages of zero, tokens without mass."""
    import torch
    x, t = _rows(1, 10, 400), torch.arange(10, device="cuda").int()
    x[5, 5], x[6, 6], x[7] = NEG, NEG, NEG
    l = binding.hbsjd_token_logprobs(x, t)[0]
    A = torch.tensor([1.0, -1.0, 0.0, 1.0, -1.0, 1.0, -2.0, 1.0, 0.0, 1.0], device="cuda")
    old = l.clone()
    old[0], old[1], old[2] = NEG, NEG, NEG         # ratio without end
    old[3], old[4] = l[3] + 500, l[4] + 500        # of zero
    old[5] = -3.0                                  # of zero, the token has no mass; 6: neither had it before
    loss, g, logp, _ = binding.hbsjd_policy_loss(x, t, A, old)
    want = [-1.2, float("inf"), 0.0, 0.0, 0.8, 0.0, 2.0, 0.0, 0.0, -1.0]
    torch.testing.assert_close(loss.cpu(), torch.tensor(want), rtol=1e-6, atol=1e-30)
    assert bool((g[0] == 0).all()) and bool((g[2:6] == 0).all()) and bool((g[7:9] == 0).all())
    assert logp[5] == NEG and logp[6] == NEG and logp[7] == NEG
    # a reference that excludes what the policy does not, and the other way
    ref = l.clone()
    ref[9], ref[5] = NEG, -3.0
    loss, g, _, _ = binding.hbsjd_policy_loss(x, t, A * 0, l, ref, kl=0.5)
    assert loss[9] == float("inf") and loss[5] == float("inf") and loss[6] == 0 and loss[0] == 0


def test_gradients_are_the_differences_of_the_loss():
    """Along random directions, by the 64-bit definition's own steps: what the tests above compare with is what autograd has."""
    import torch
    g = _gen(3)
    x = _rows(4, 6, 60).double().requires_grad_()
    t = sampled(x.detach(), 1.0, g)
    logq = torch.log_softmax(x / 0.8, -1)
    l = logq.gather(1, t.long()[:, None])[:, 0]
    H = -(logq.exp() * logq).sum(-1)
    A, old, ref = (torch.randn(6, generator=g, device="cuda").double() for _ in range(3))
    old, ref = l.detach() - old * 0.3, l.detach() - ref * 0.3
    ratio = (l - old).exp()
    loss = -torch.min(ratio * A, ratio.clamp(0.8, 1.2) * A) + 0.1 * ((ref - l).exp() - 1 - (ref - l)) - 0.05 * H
    loss.sum().backward()
    got = binding.hbsjd_policy_loss(x.detach().float(), t, A.float(), old.float(), ref.float(), temperature=0.8, kl=0.1, entropy=0.05)
    torch.testing.assert_close(got[1].double(), x.grad, rtol=2e-4, atol=2e-6)
    y = x.detach().float()
    d = torch.randn(6, 60, generator=g, device="cuda")
    run = lambda s: binding.hbsjd_policy_loss((y.double() + s * d.double()).float(), t, A.float(), old.float(), ref.float(), temperature=0.8,
                                              kl=0.1, entropy=0.05, want_grad=False)[0].double()
    h = 2e-3  # (rounded losses: 2e-7 / h; the third derivative's h^2)
    slope = (run(h) - run(-h)) / (2 * h)
    torch.testing.assert_close(slope, (got[1] * d).double().sum(-1), rtol=5e-3, atol=2e-3)


def test_streams_devices_and_autograd():
    import torch
    x, t = _rows(1, 50, 3000), torch.arange(50, device="cuda").int()
    A = torch.ones(50, device="cuda")
    want = binding.hbsjd_policy_loss(x, t, A, entropy=0.01)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = binding.hbsjd_policy_loss(x, t, A, entropy=0.01, stream=side)
    lp = binding.hbsjd_token_logprobs(x, t, stream=side)
    bw = binding.hbsjd_token_logprobs_grad(x, t, A, A, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    assert torch.equal(lp[0], want[2]) and torch.equal(bw, binding.hbsjd_token_logprobs_grad(x, t, A, A))
    y = x.clone().requires_grad_()
    logits = y.tanh()
    binding.hbsjd_policy_loss(logits.detach(), t, A, grad=logits.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logits.backward(torch.ones_like(logits))


def test_captured_and_replayed():
    import torch
    x, t = _rows(1, 300, 5000), torch.randint(0, 5000, (300,), device="cuda").int()
    A, old = torch.randn(300, device="cuda"), torch.full((300,), -8.0, device="cuda")
    binding.hbsjd_policy_loss(x, t, A, old)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, g, logp, _ = binding.hbsjd_policy_loss(x, t, A, old, kl=0.1, ref_logp=old, entropy=0.1)
    for seed in (5, 6):
        x.copy_(_rows(seed, 300, 5000))
        graph.replay()
        want = binding.hbsjd_policy_loss(x, t, A, old, kl=0.1, ref_logp=old, entropy=0.1)
        assert torch.equal(loss, want[0]) and torch.equal(g, want[1]) and torch.equal(logp, want[2])


def test_refusals_of_tensors():
    import torch
    x, t, A = _rows(1, 4, 50), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(4, device="cuda")
    for call in (lambda: binding.hbsjd_token_logprobs(x, t.long()), lambda: binding.hbsjd_token_logprobs(x, t[:3]),
                 lambda: binding.hbsjd_token_logprobs(x, None), lambda: binding.hbsjd_token_logprobs(x.half(), t),
                 lambda: binding.hbsjd_token_logprobs(x.t(), t), lambda: binding.hbsjd_token_logprobs(x, t.cpu()),
                 lambda: binding.hbsjd_token_logprobs(x, t, 0.0), lambda: binding.hbsjd_token_logprobs_grad(x, t, None),
                 lambda: binding.hbsjd_token_logprobs_grad(x, t, A, A.double()),
                 lambda: binding.hbsjd_token_logprobs_grad(x, t, A, grad=x.bfloat16()),
                 lambda: binding.hbsjd_policy_loss(x, t, None), lambda: binding.hbsjd_policy_loss(x, t, A, kl=0.1),
                 lambda: binding.hbsjd_policy_loss(x, t, A, clip_low=1.5), lambda: binding.hbsjd_policy_loss(x, t, A, dual_clip=0.5),
                 lambda: binding.hbsjd_policy_loss(x, t, A, grad=torch.empty(4, 51, device="cuda"))):
        with pytest.raises(binding.HbsjdError) as e:
            call()
        assert e.value.code == -1


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_large_factors_beside_masked_entries(dtype):
    """Slopes and weights of up to 1e20: no entry without mass has a gradient."""
    import torch
    x = _rows(5, 6, 2000, 3.0, dtype)
    x[:, ::3] = NEG
    x[3:, 1::3] = -1e30
    t = torch.full((6,), 2, dtype=torch.int32, device="cuda")
    for size in (1e8, 1e15, 1e20):
        a = torch.full((6,), size, device="cuda")
        for ent in (None, a, -a):
            r = Rows(x, t, 0.5)
            g = binding.hbsjd_token_logprobs_grad(x, t, a, ent, 0.5)
            want, bound = r.gradient(a.double(), None if ent is None else ent.double(), torch.ones_like(r.l))
            near(g, want, bound, HALF[dtype])
            assert not bool(g[:, ::3].any())


def test_slopes_that_are_no_numbers():
    """NaN slopes make their row's gradient NaN, where the token has all the mass too."""
    import torch
    x, t = _rows(5, 4, 300), torch.full((4,), 7, dtype=torch.int32, device="cuda")
    x[1] = NEG
    x[1, 7] = 1.0
    a = torch.tensor([1.0, float("nan"), float("nan"), 1.0], device="cuda")
    for ent in (None, a):
        g = binding.hbsjd_token_logprobs_grad(x, t, a, ent)
        assert bool(torch.isnan(g[1:3]).all()) and bool(torch.isfinite(g[0]).all()) and bool(torch.isfinite(g[3]).all())


def test_places_beyond_32_bits():
    """More than 2^32 bytes and 2^31 entries of logits: the last rows are as they are alone."""
    import torch
    rows, V = 132000, 16384
    x = torch.zeros(rows, V, dtype=torch.bfloat16, device="cuda")
    t = torch.randint(0, V, (rows,), generator=_gen(1), device="cuda").int()
    x[-300:] = _rows(2, 300, V, 3.0, "bf16")
    A = torch.randn(rows, generator=_gen(3), device="cuda")
    loss, g, logp, _ = binding.hbsjd_policy_loss(x, t, A, entropy=0.01)
    alone = binding.hbsjd_policy_loss(x[-300:], t[-300:], A[-300:], entropy=0.01)
    # (other CTAs, other orders of a row's sums)
    torch.testing.assert_close(loss[-300:], alone[0], rtol=1e-5, atol=1e-6)
    torch.testing.assert_close(logp[-300:], alone[2], rtol=1e-5, atol=1e-6)
    torch.testing.assert_close(g[-300:].float(), alone[1].float(), rtol=1e-2, atol=1e-9)
    flat = torch.tensor(V, device="cuda").double().log()
    near(logp[:-300], -flat.expand(rows - 300), torch.full_like(logp[:-300], 2e-5).double(), HALF["fp32"])
    offsets = torch.tensor([0, rows - 300, rows - 150, rows - 150, rows], device="cuda").int()
    small = torch.tensor([0, 0, 150, 150, 300], device="cuda").int()
    _, g2, sums = binding.hbsjd_preference_loss(x, t, offsets, beta=1e-4, grad=g)
    _, want, wsums = binding.hbsjd_preference_loss(x[-300:], t[-300:], small, beta=1e-4)
    torch.testing.assert_close(sums[1:], wsums[1:], rtol=1e-5, atol=1e-4)
    assert bool(torch.isfinite(g2[-150:]).all()) and bool((g2[-150:].float().abs().sum(-1) > 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_long_rows_out_of_the_ordinary(dtype):
    """More rows than SMs, each longer than a CTA holds: parts without mass, the token in any of them, maxima at either end."""
    import torch
    V, rows = 60001, 330
    x = _rows(7, rows, V, 3.0, dtype, 1)
    t = sampled(x, 1.0, _gen(7))
    kind = torch.arange(rows, device="cuda") % 11
    x[kind == 1, :30000] = NEG
    x[kind == 2, 20000:] = NEG
    x[kind == 3] = NEG
    x[kind == 4] = NEG
    x[kind == 4, 41234] = 2.0
    t[kind == 4] = 41234
    x[kind == 5, 59999] = 60.0
    x[kind == 6, 3] = 60.0
    x[kind == 7] -= 5000.0
    t[kind == 8] = 60000
    t[kind == 9] = 0
    t[kind == 10] = -1
    x[kind == 10] = float("nan")
    live = kind != 10
    r = Rows(x[live], t[live], 1.0)
    logp, H = binding.hbsjd_token_logprobs(x, t)
    near(logp[live], r.l, r.dl, HALF["fp32"])
    near(H[live], r.H, r.dH, HALF["fp32"])
    assert not bool(logp[~live].any()) and not bool(H[~live].any())
    assert torch.equal(binding.hbsjd_token_logprobs(x, t, want_entropy=False)[0].isinf(), logp.isinf())


def test_nan_advantages_and_weights_reach_every_entry():
    import torch
    x, t = _rows(1, 6, 3000) * 40, torch.ones(6, dtype=torch.int32, device="cuda")
    x[:, ::7] = NEG
    one = torch.ones(6, device="cuda")
    bad = one.clone()
    bad[2] = float("nan")
    for call in (lambda ent: binding.hbsjd_policy_loss(x, t, bad, entropy=ent), lambda ent: binding.hbsjd_policy_loss(x, t, one, bad, entropy=ent),
                 lambda ent: binding.hbsjd_policy_loss(x, t, one, weight=bad, entropy=ent),
                 lambda ent: binding.hbsjd_policy_loss(x, t, one, ref_logp=bad, kl=0.1, entropy=ent)):
        for ent in (0.0, 0.1):
            g = call(ent)[1]
            # (against a reference of e^1, tokens of e^-400 have slopes beyond fp32: infinite, no NaN)
            assert bool(torch.isnan(g[2]).all()) and not bool(torch.isnan(g[[0, 1, 3, 4, 5]]).any())


def test_host_threads_and_streams_at_once():
    import threading
    import torch
    x, t = _rows(1, 333, 5001), torch.randint(0, 5001, (333,), generator=_gen(1), device="cuda").int()
    A, offsets = torch.randn(333, generator=_gen(2), device="cuda"), torch.tensor([0, 100, 150, 300, 333], device="cuda").int()
    arrays = [torch.randn(n, generator=_gen(n), device="cuda") for n in (100000, 33, 70001)]
    outs = [torch.empty_like(v) for v in arrays]

    def calls(out):
        p = binding.hbsjd_policy_loss(x, t, A, entropy=0.01)
        q = binding.hbsjd_preference_loss(x, t, offsets)
        n = binding.hbsjd_clip_gradients(arrays, 3.0, out=out)
        return [*p[:3], *q, *binding.hbsjd_token_logprobs(x, t), n, *out]

    want = [v.clone() for v in calls(outs)]
    torch.cuda.synchronize()
    wrong = []

    def work():
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            own = [torch.empty_like(v) for v in arrays]
            for _ in range(30):
                got = calls(own)
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append(1)
            stream.synchronize()

    threads = [threading.Thread(target=work) for _ in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not wrong
