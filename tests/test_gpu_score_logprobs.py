"""hbsjd_score_logprobs: a model's log-probabilities over finished trajectories, against the oracle's logits and hbsjd_score_topk, and the
runs that they are made for: rollout, old policy and reference, the student's loss, gradients and their clipping."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2608_18183_b200 import binding, synth
from tests import gpu_util as G
from tests.test_gpu_score_topk import _inputs, _logits

pytestmark = pytest.mark.gpu


def test_of_an_fp32_model_are_the_oracle_s():
    w = synth.WORKLOADS["tiny"]
    T = w.shape.T
    toks, k, lab = _inputs(w, 1, [0, 13, T - 1, T, 40])
    ctx = binding.Context(w.shape, G.weights_for(w), 6, w.window)
    model = O.Model(w.shape, G.weights_for(w))
    for tau in (1.0, 0.7):
        logp, H = (x.cpu().numpy() for x in ctx.hbsjd_score_logprobs(G.dev(toks), G.dev(k), G.dev(lab), tau))
        for b in range(len(k)):
            assert (logp[b, :k[b]] == 0).all() and (H[b, :k[b]] == 0).all()
            if k[b] == T:
                continue
            seq = np.concatenate([[0], toks[b, :T - 1]]).astype(np.int32)
            l = model.forward_full(int(lab[b]), seq)[k[b]:].astype(np.float64) / tau
            lq = l - np.log(np.exp(l - l.max(1, keepdims=True)).sum(1, keepdims=True)) - l.max(1, keepdims=True)
            # fp32 forwards of both sides: 1e-4 on logits of size 10, as the forward tests hold them to
            np.testing.assert_allclose(logp[b, k[b]:], np.take_along_axis(lq, toks[b, k[b]:, None].astype(int), 1)[:, 0], rtol=2e-4, atol=2e-4)
            np.testing.assert_allclose(H[b, k[b]:], -(np.exp(lq) * lq).sum(1), rtol=5e-4, atol=5e-4)
    ctx.hbsjd_destroy()


@pytest.mark.parametrize("name", ["tiny", "tiny_bf16", "small_bf16"])
def test_of_the_lists_logits(name):
    """What hbsjd_token_logprobs has of the logits that lists of the whole vocabulary give."""
    import torch
    w = synth.WORKLOADS[name]
    V, T = w.shape.vocab, w.shape.T
    toks, k, lab = _inputs(w, 2, [0, 5, T // 2, T - 1, T])
    ctx = binding.Context(w.shape, G.weights_for(w), len(k), w.window)
    args = G.dev(toks), G.dev(k), G.dev(lab)
    logp, H = ctx.hbsjd_score_logprobs(*args)
    logits, live = _logits(ctx.hbsjd_score_topk(*args, V), V)
    want, wantH = binding.hbsjd_token_logprobs(logits, args[0].reshape(-1))
    # (the order of a row's sums may depend on how many rows there are)
    torch.testing.assert_close(logp.reshape(-1)[live], want[live], rtol=2e-6, atol=2e-6)
    torch.testing.assert_close(H.reshape(-1)[live], wantH[live], rtol=5e-6, atol=5e-6)
    assert not bool(logp.reshape(-1)[~live].any()) and not bool(H.reshape(-1)[~live].any())
    again = ctx.hbsjd_score_logprobs(*args)
    assert torch.equal(again[0], logp) and torch.equal(again[1], H)
    ctx.hbsjd_destroy()


def test_refusals():
    w = synth.WORKLOADS["tiny"]
    T = w.shape.T
    ctx = binding.Context(w.shape, G.weights_for(w), 4, w.window)
    good = dict(zip("tkl", _inputs(w, 1, [0, 3])))
    for change in (dict(k=np.array([0, T + 1], np.int32)), dict(k=np.array([-1, 0], np.int32)), dict(l=np.array([0, 11], np.int32)),
                   dict(t=np.where(np.arange(T) == 5, w.shape.vocab, good["t"]).astype(np.int32))):
        a = {**good, **change}
        with pytest.raises(binding.HbsjdError) as e:
            ctx.hbsjd_score_logprobs(G.dev(a["t"]), G.dev(a["k"]), G.dev(a["l"]))
        assert e.value.code == -1
    with pytest.raises(binding.HbsjdError):
        ctx.hbsjd_score_logprobs(*(G.dev(good[n]) for n in "tkl"), temperature=0.0)
    five = _inputs(w, 1, [0, 3, 0, 0, 0])
    with pytest.raises(binding.HbsjdError):
        ctx.hbsjd_score_logprobs(*(G.dev(x) for x in five))
    ctx.hbsjd_destroy()


class _Student:
    """A model of one matrix a token: logits of position t from token t - 1 (the first from the class)."""

    def __init__(self, V, C, D, seed):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda *s: torch.randn(*s, generator=g, device="cuda").mul_(0.2).requires_grad_()
        self.tok, self.cls, self.head = make(V, D), make(C + 1, D), make(V, D)
        self.parameters = [self.tok, self.cls, self.head]

    def __call__(self, tokens, labels):
        import torch
        h = torch.cat([self.cls[labels.long()][:, None], self.tok[tokens[:, :-1].long()]], 1)
        return (h @ self.head.t()).reshape(-1, self.head.shape[0])


def _step(kind, graph=False):
    """A step of training on rollouts: losses and parameters' gradients by the operators, and by torch in 64 bits."""
    import torch
    w = synth.WORKLOADS["tiny"]
    T, V, B = w.shape.T, w.shape.vocab, 4
    toks, k, lab = _inputs(w, 3, [0, 5, 20, 2])
    ctx = binding.Context(w.shape, G.weights_for(w), B, w.window)
    ref_ctx = binding.Context(w.shape, synth.make_weights(w.shape, 91), B, w.window)
    tokens, _ = ctx.hbsjd_rollout(G.dev(toks), G.dev(k), G.dev(lab), G.gpu_params(w, 7))
    args = tokens, G.dev(k), G.dev(lab)
    old, ref = ctx.hbsjd_score_logprobs(*args)[0].view(-1), ref_ctx.hbsjd_score_logprobs(*args)[0].view(-1)
    ctx.hbsjd_destroy()
    ref_ctx.hbsjd_destroy()
    student = _Student(V, w.shape.n_classes, 32, 5)
    flat, labels = tokens.reshape(-1), G.dev(lab)
    live = (torch.arange(T, device="cuda")[None] >= G.dev(k)[:, None]).float().reshape(-1)
    weight = live / live.sum()
    reward = torch.tensor([1.0, -0.5, 0.3, -0.8], device="cuda").repeat_interleave(T)
    offsets = torch.arange(B + 1, device="cuda").int() * T
    logits = student(tokens, labels)
    if kind == "policy":
        loss, grad, _, _ = binding.hbsjd_policy_loss(logits.detach(), flat, reward, old, ref, weight, kl=0.05, entropy=0.01)
        total = (loss * weight).sum()
    else:
        loss, grad, _ = binding.hbsjd_preference_loss(logits.detach(), flat, offsets, ref, live, beta=0.1, interleaved=True)
        total = loss.sum()
    logits.backward(grad)
    own = [p.grad for p in student.parameters]
    raw = [g.clone() for g in own]
    limit = 0.5 * float(torch.sqrt(sum(g.double().square().sum() for g in own)))
    norm = binding.hbsjd_clip_gradients(own, limit)
    # the same in 64 bits
    twin = _Student(V, w.shape.n_classes, 32, 5)
    for p, q in zip(twin.parameters, student.parameters):
        p.data = q.data.double()
        p.requires_grad_()
    logq = torch.log_softmax(twin(tokens, labels), -1)
    l = logq.gather(1, flat.long()[:, None])[:, 0]
    if kind == "policy":
        r = (l - old.double()).exp()
        A = reward.double()
        d = ref.double() - l
        H = -(logq.exp() * logq).sum(-1)
        want = ((-torch.min(r * A, r.clamp(0.8, 1.2) * A) + 0.05 * (d.exp() - 1 - d) - 0.01 * H) * weight.double()).sum()
    else:
        S = ((l - ref.double()) * live.double()).view(B, T).sum(1)
        want = -torch.nn.functional.logsigmoid(0.1 * (S[0::2] - S[1::2])).sum()
    want.backward()
    return total, want, raw, [p.grad for p in twin.parameters], own, norm, limit


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_a_step_on_rollouts(kind):
    import torch
    total, want, raw, exact, clipped, norm, limit = _step(kind)
    want = want.detach()
    # log-probabilities within 5e-5 (rounded logits), summed over a sequence for a pair
    assert abs(float(total) - float(want)) <= 2e-4 * abs(float(want)) + 1e-6
    for g, e in zip(raw, exact):
        assert float((g.double() - e).norm()) <= 1e-3 * float(e.norm())
    size = float(torch.sqrt(sum(e.square().sum() for e in exact)))
    assert abs(float(norm) - size) <= 1e-3 * size
    for c, g in zip(clipped, raw):
        torch.testing.assert_close(c, g * (limit / (float(norm) + 1e-6)), rtol=1e-5, atol=0)


def test_a_step_captured_into_a_graph():
    """Loss, gradient, backward and clipping as one graph, replayed on new tokens."""
    import torch
    V, T, B = 500, 16, 4
    student = _Student(V, 3, 24, 1)
    tokens = torch.randint(0, V, (B, T), device="cuda").int()
    labels, A, old = torch.zeros(B, device="cuda").int(), torch.randn(B * T, device="cuda"), torch.full((B * T,), -6.3, device="cuda")
    weight = torch.full((B * T,), 1.0 / (B * T), device="cuda")
    for p in student.parameters:
        p.grad = torch.zeros_like(p)

    def step():
        for p in student.parameters:
            p.grad.zero_()
        logits = student(tokens, labels)
        loss, grad, _, _ = binding.hbsjd_policy_loss(logits.detach(), tokens.view(-1), A, old, weight=weight, entropy=0.01)
        logits.backward(grad)
        return loss, binding.hbsjd_clip_gradients([p.grad for p in student.parameters], 1e-3)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm = step()
    for seed in (1, 2):
        tokens.copy_(torch.randint(0, V, (B, T), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [loss.clone(), norm.clone()] + [p.grad.clone() for p in student.parameters]
        want = list(step()) + [p.grad for p in student.parameters]
        for g, w in zip(got, want):
            torch.testing.assert_close(g, w, rtol=1e-4, atol=1e-9)
