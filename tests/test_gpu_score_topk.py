"""hbsjd_score_topk: a model's lists over finished trajectories, against the oracle's logits and against hbsjd_score, and the run
that they are made for: rollout, the teacher's lists, the student's loss and gradient."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2608_18183_b200 import binding, synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu


def _teacher_shape(s):
    """A wider, deeper model over the same vocabulary, grid and classes."""
    return synth.ModelShape(s.n_layers + 1, s.dim * 2, s.n_heads * 2, s.ffn_hidden * 2, s.vocab, s.grid_h, s.grid_w,
                            s.n_classes, s.dtype)


def _inputs(w, seed, k):
    rng = np.random.default_rng(seed)
    toks = rng.integers(0, w.shape.vocab, size=(len(k), w.shape.T)).astype(np.int32)
    lab = rng.integers(0, w.shape.n_classes, size=len(k)).astype(np.int32)
    return toks, np.array(k, dtype=np.int32), lab


def _logits(lists, V):
    """[B * T, V] logits again from lists of all V entries; rows of empty lists are zeros."""
    import torch
    values, indices, rest = lists
    flat = indices.reshape(-1, V).long()
    empty = flat[:, 0] < 0
    out = torch.zeros(flat.shape, device="cuda")
    out.scatter_(1, flat.clamp(min=0), torch.where(empty[:, None], 0.0, values.reshape(-1, V)))
    assert bool((rest == float("-inf")).all())
    return out, ~empty


def test_lists_of_an_fp32_model_are_the_oracle_s():
    w = synth.WORKLOADS["tiny"]
    T, V = w.shape.T, w.shape.vocab
    toks, k, lab = _inputs(w, 1, [0, 13, T - 1, T, 40])
    ctx = binding.Context(w.shape, G.weights_for(w), 6, w.window)
    model = O.Model(w.shape, G.weights_for(w))
    for K in (1, 20, V):
        values, indices, rest = (x.cpu().numpy() for x in ctx.hbsjd_score_topk(G.dev(toks), G.dev(k), G.dev(lab), K, 0.8))
        for b in range(len(k)):
            assert (indices[b, :k[b]] == -1).all() and np.isneginf(values[b, :k[b]]).all() and np.isneginf(rest[b, :k[b]]).all()
            if k[b] == T:
                continue
            seq = np.concatenate([[0], toks[b, :T - 1]]).astype(np.int32)
            l = model.forward_full(int(lab[b]), seq)[k[b]:].astype(np.float64)
            # fp32 forwards of both sides: 1e-4 on logits of size 10, as the forward tests hold them to
            at = indices[b, k[b]:]
            np.testing.assert_allclose(values[b, k[b]:], np.take_along_axis(l, at.astype(int), 1), rtol=1e-4, atol=1e-4)
            top = -np.sort(-l, axis=1)
            np.testing.assert_allclose(values[b, k[b]:], top[:, :K], rtol=1e-4, atol=1e-4)
            if K < V:
                others = l.copy()
                np.put_along_axis(others, at.astype(int), -np.inf, 1)
                m = others.max(1, keepdims=True)
                want = np.log(np.exp((others - m) / 0.8).sum(1)) + m[:, 0] / 0.8
                np.testing.assert_allclose(rest[b, k[b]:], want, rtol=2e-4, atol=2e-4)
            else:
                assert np.isneginf(rest[b, k[b]:]).all()
    ctx.hbsjd_destroy()


@pytest.mark.parametrize("name", ["tiny", "small_bf16"])
def test_lists_of_everything_give_the_score(name):
    """With lists as long as the vocabulary, hbsjd_distill on both models' logits is what hbsjd_score computes position by position
    (the same forwards; sums of V terms in another order)."""
    import torch
    w = synth.WORKLOADS[name]
    V, T = w.shape.vocab, w.shape.T
    toks, k, lab = _inputs(w, 2, [0, 5, T // 2, T - 1, T])
    tsh = _teacher_shape(w.shape)
    stu = binding.Context(w.shape, G.weights_for(w), len(k), w.window)
    tea = binding.Context(tsh, synth.make_weights(tsh, 77), len(k), w.window)
    args = G.dev(toks), G.dev(k), G.dev(lab)
    pos, per, loss = stu.hbsjd_score(tea, *args)
    s, live = _logits(stu.hbsjd_score_topk(*args, V), V)
    t, live_t = _logits(tea.hbsjd_score_topk(*args, V), V)
    assert torch.equal(live, live_t)
    row, _ = binding.hbsjd_distill(s, t, live.float(), want_grad=False)
    want = pos.reshape(-1)
    assert bool(((row - want).abs() <= 1e-4 * (1 + want)).all()) and float(want.max()) > 0.05
    # the same again: neither call leaves anything behind for the other
    again = stu.hbsjd_score(tea, *args)
    assert torch.equal(again[0], pos) and again[2] == loss
    stu.hbsjd_destroy()
    tea.hbsjd_destroy()


def test_rollout_lists_loss_and_gradient():
    """One step as the loop makes it: the student samples, the teacher's lists are stored, the student's logits at the same positions
    get loss and gradient; prefixes take no part.  Against 64 bits."""
    import torch
    w = synth.WORKLOADS["small_bf16"]
    V, T, K = w.shape.vocab, w.shape.T, 100
    weights = G.weights_for(w)
    toks, k, lab = synth.make_inputs(w)
    stu = binding.Context(w.shape, weights, w.batch, w.window)
    tsh = _teacher_shape(w.shape)
    tea = binding.Context(tsh, synth.make_weights(tsh, 77), w.batch, w.window)
    p = binding.make_params(w.window, w.history_offset, w.cfg_scale, w.temperature, w.top_k, binding.VERIFY_PROB,
                            binding.EXEC_HYBRID, w.batch // 2, 3, -1)
    out, _ = stu.hbsjd_rollout(G.dev(toks), G.dev(k), G.dev(lab), p)
    values, indices, rest = tea.hbsjd_score_topk(out, G.dev(k), G.dev(lab), K)
    s, live = _logits(stu.hbsjd_score_topk(out, G.dev(k), G.dev(lab), V), V)
    weight = live.float() / int(live.sum())
    for dtype in (torch.float32, torch.bfloat16):
        x = s.to(dtype)
        loss, grad = binding.hbsjd_distill_topk(x, values.view(-1, K), indices.view(-1, K), rest.view(-1), weight, 1.0, 0.5, 0.5)
        # empty lists alone leave the prefixes out, too
        bare = binding.hbsjd_distill_topk(x, values.view(-1, K), indices.view(-1, K), rest.view(-1), None, 1.0, 0.5, 0.5)
        assert torch.equal(bare[0], loss) and not bool(bare[1][~live].any()) and not bool(grad[~live].any())
        l64 = x[live].double().requires_grad_()
        idx = indices.view(-1, K)[live].long()
        lq = torch.log_softmax(l64, -1)
        o = torch.logsumexp(lq.scatter(1, idx, float("-inf")), -1, keepdim=True)
        lq = torch.cat([lq.gather(1, idx), o], 1)
        lp = torch.log_softmax(torch.cat([values.view(-1, K), rest.view(-1, 1)], 1)[live].double(), -1)
        rows = 0.5 * (lp.exp() * (lp - lq)).sum(-1) + 0.5 * (lq.exp() * (lq - lp)).sum(-1)
        rows.mean().backward()
        assert bool(((loss[live].double() - rows.detach()).abs() <= 5e-5 * (1 + rows.detach())).all())
        tol = 5e-5 * (l64.grad.abs() + l64.grad.abs().amax(-1, keepdim=True)) + (2.0 ** -8 if dtype == torch.bfloat16 else 0) * l64.grad.abs()
        assert bool(((grad[live].double() - l64.grad).abs() <= tol).all())
    stu.hbsjd_destroy()
    tea.hbsjd_destroy()


def test_refusals():
    import torch
    w = synth.WORKLOADS["tiny"]
    T, V = w.shape.T, w.shape.vocab
    ctx = binding.Context(w.shape, G.weights_for(w), 2, w.window)
    toks, k, lab = _inputs(w, 5, [3, 9])
    def call(t=toks, kk=k, ll=lab, K=5, tau=1.0):
        return ctx.hbsjd_score_topk(G.dev(t), G.dev(kk), G.dev(ll), K, tau)
    bad = toks.copy()
    bad[1, 7] = V
    for kw in (dict(t=bad), dict(kk=np.array([3, T + 1], np.int32)), dict(ll=np.array([-1, 0], np.int32)), dict(K=0), dict(K=V + 1),
               dict(tau=0.0), dict(tau=float("nan")),
               dict(t=np.zeros((3, T), np.int32), kk=np.zeros(3, np.int32), ll=np.zeros(3, np.int32))):
        with pytest.raises(binding.HbsjdError) as e:
            call(**kw)
        assert e.value.code == -1
    a, b = call(), call()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    ctx.hbsjd_destroy()
