"""Training on a model's own rollouts by rewards and preferences, as measurable cases through the public entry points.

What a step on finished trajectories does when there is no teacher, next to the divergences of the distillation step:

  logprobs      hbsjd_token_logprobs: log-probability of every sampled token and the entropy of its distribution (the old policy's
                and the reference's sides of the losses); backward: hbsjd_token_logprobs_grad, for losses of a user's own.
  policy        hbsjd_policy_loss: the clipped policy loss with a KL term and an entropy bonus, and its gradient.
  preference    hbsjd_preference_loss: a loss of paired log ratios over whole sequences, and its gradient.
  clip          hbsjd_clip_gradients: the global norm of all gradients, and clipping by it.

Sizes: the vocabulary of 16384 image tokens, 256 positions an image and the decoder's widths are the library's own L and B
workloads; vocabularies of 1000 to 65537 entries stand for other tokenizers, odd ones for rows that are not aligned.
"""
from __future__ import annotations

import math

import torch

own = False

_T = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2}
_POSITIONS = 256  # positions of an image: rows are (image, position) pairs


# ------------------------------------------------------------------ cases
def _logprobs(rows, vocab, dtype, temperature, entropy, backward, masked, pad):
    return dict(op="logprobs", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, entropy=entropy, backward=backward,
                masked=masked, pad=pad)


def _policy(rows, vocab, dtype, temperature, low, high, dual, kl, entropy, old, grad, prefix, pad):
    return dict(op="policy", rows=rows, vocab=vocab, dtype=dtype, temperature=temperature, low=low, high=high, dual=dual, kl=kl,
                entropy=entropy, old=old, grad=grad, prefix=prefix, pad=pad)


def _preference(pairs, length, ragged, vocab, dtype, kind, beta, smoothing, margin, reference, mean, interleaved, grad, prefix, pad):
    return dict(op="preference", pairs=pairs, length=length, ragged=ragged, vocab=vocab, dtype=dtype, kind=kind, beta=beta,
                smoothing=smoothing, margin=margin, reference=reference, mean=mean, interleaved=interleaved, grad=grad,
                prefix=prefix, pad=pad)


def _clip(layers, dim, ffn, vocab, dtype, norm, clipped, align):
    return dict(op="clip", layers=layers, dim=dim, ffn=ffn, vocab=vocab, dtype=dtype, norm=norm, clipped=clipped, align=align)


def listed():
    return [
        # the tokens that one image's window has just committed
        dict(name="logprobs_few", **_logprobs(32, 16384, "fp32", 1.0, True, False, False, 0)),
        # a batch's positions under the reference model
        dict(name="logprobs_batch", **_logprobs(8192, 16384, "fp32", 1.0, True, False, False, 0)),
        # a loss of the user's own over a vocabulary of text and images: bf16 rows that are not aligned, a tenth masked
        dict(name="logprobs_backward_odd_bf16", **_logprobs(3001, 24001, "bf16", 0.8, True, True, True, 0)),
        # a few positions, on-policy: the ratio is one
        dict(name="policy_few", **_policy(37, 16384, "fp32", 1.0, 0.2, 0.2, 0.0, 0.0, 0.0, False, True, 0, 0)),
        # a batch's positions with clipping and the KL term; the first 32 positions of every image are its real prefix
        dict(name="policy_batch", **_policy(16384, 16384, "fp32", 1.0, 0.2, 0.28, 0.0, 0.04, 0.0, True, True, 32, 0)),
        # every term on, bf16 logits
        dict(name="policy_entropy_bf16", **_policy(8192, 16384, "bf16", 1.0, 0.2, 0.2, 3.0, 0.02, 0.01, True, True, 0, 0)),
        # one pair of short sequences
        dict(name="preference_few", **_preference(1, 24, False, 16384, "fp32", "sigmoid", 0.1, 0.0, 0.0, True, False, False, True, 0, 0)),
        # sixteen pairs of images, preferred first in the batch; their real prefixes are left out
        dict(name="preference_batch",
             **_preference(16, 256, False, 16384, "fp32", "sigmoid", 0.1, 0.1, 0.0, True, False, False, True, 32, 0)),
        # pairs of texts of any length, means over positions and no reference, a wide bf16 vocabulary
        dict(name="preference_ragged_bf16",
             **_preference(24, 400, True, 32768, "bf16", "sigmoid", 2.0, 0.0, 0.5, False, True, True, True, 0, 0)),
        # the gradients of a small decoder
        dict(name="clip_small", **_clip(2, 256, 512, 1024, "fp32", "2", True, 64)),
        # those of the L student in fp32, into the optimizer's buffers
        dict(name="clip_model", **_clip(24, 1024, 2816, 16384, "fp32", "2", True, 64)),
        # those of the B student in bf16, in place, below the limit: nothing is to be scaled
        dict(name="clip_below_bf16", **_clip(12, 768, 2048, 16384, "bf16", "2", False, 64)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "policy", "policy", "preference", "preference", "clip"])
    vocab = rng.choice([16384, 16384, _log_int(rng, 1000, 65537), _log_int(rng, 1000, 65537)])
    dtype = rng.choice(["fp32", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 64])  # rows of a wider buffer
    cap = 8192 * 16384 // 2             # elements of a drawn case, at most
    rows = _log_int(rng, 1, max(2, min(16384, cap // vocab)))
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
    if op == "logprobs":
        return _logprobs(rows, vocab, dtype, temperature, rng.random() < 0.7, rng.random() < 0.5, rng.random() < 0.3, pad)
    if op == "policy":
        low, high = rng.choice([(0.2, 0.2), (0.2, 0.28), (0.1, 0.1)])
        return _policy(rows, vocab, dtype, temperature, low, high, rng.choice([0.0, 0.0, 3.0]), rng.choice([0.0, 0.04, 0.1]),
                       rng.choice([0.0, 0.0, 0.01]), rng.random() < 0.8, rng.random() < 0.8, min(rng.choice([0, 0, 17, 64]), rows // 2),
                       pad)
    if op == "preference":
        length = _log_int(rng, 1, 1024)
        pairs = _log_int(rng, 1, max(1, min(64, cap // (2 * length * vocab))))
        kind = rng.choice(["sigmoid", "sigmoid", "hinge", "square"])
        return _preference(pairs, length, rng.random() < 0.5, vocab, dtype, kind, rng.choice([0.1, 0.3, 1.0]),
                           rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0, rng.choice([0.0, 0.5]) if kind != "square" else 0.0,
                           rng.random() < 0.7, rng.random() < 0.3, rng.random() < 0.5, rng.random() < 0.85,
                           min(rng.choice([0, 0, 17]), length // 2), pad)
    return _clip(rng.randint(1, 24), _log_int(rng, 33, 1024), _log_int(rng, 65, 2816), _log_int(rng, 256, 16384),
                 rng.choice(["fp32", "bf16", "mixed"]), rng.choice(["2", "2", "max"]), rng.random() < 0.7, rng.choice([64, 64, 1]))


# ------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(c, rows, g, scale):
    """[rows, vocab] logits, a view of wider rows where the case has padding."""
    buf = torch.randn(rows, c["vocab"] + c["pad"], generator=g, device="cuda")
    return buf.mul_(scale).to(_T[c["dtype"]])[:, :c["vocab"]]


def _sampled(x, temperature, g):
    """A token of every row by its distribution, and its log-probability."""
    tokens, logp = [], []
    for part in x.split(1024):
        y = part.float() / temperature
        noise = torch.rand(y.shape, generator=g, device="cuda").clamp_(min=1e-30).log_().neg_().log_().neg_()
        t = noise.add_(y).argmax(-1)
        tokens.append(t.int())
        logp.append(y.gather(1, t[:, None])[:, 0] - torch.logsumexp(y, -1))
    return torch.cat(tokens), torch.cat(logp)


def _left_out(c):
    return c["rows"] // _POSITIONS * c["prefix"] + min(c["rows"] % _POSITIONS, c["prefix"])


def _prepare_logprobs(c, g):
    x = _matrix(c, c["rows"], g, 3.0)
    if c["masked"]:
        x[:, torch.rand(c["vocab"], generator=g, device="cuda") < 0.1] = float("-inf")
    tokens, _ = _sampled(x, c["temperature"], g)
    st = dict(logits=x, tokens=tokens)
    if c["backward"]:
        st["d_logp"] = torch.randn(c["rows"], generator=g, device="cuda") / c["rows"]
        st["d_entropy"] = torch.randn(c["rows"], generator=g, device="cuda") * (0.01 / c["rows"]) if c["entropy"] else None
    return st


def _prepare_policy(c, g):
    rows = c["rows"]
    x = _matrix(c, rows, g, 3.0)
    tokens, logp = _sampled(x, c["temperature"], g)
    at = torch.arange(rows, device="cuda") % _POSITIONS
    weight = torch.where(at < c["prefix"], 0.0, 1.0 / max(1, rows - _left_out(c))).float()
    # one advantage an image; the policy has moved a little since the rollout, the reference is further away
    image = torch.arange(rows, device="cuda") // _POSITIONS
    advantage = torch.randn(int(image[-1]) + 1, generator=g, device="cuda")[image]
    ratio = torch.randn(rows, generator=g, device="cuda") * 0.15
    for border in (1 - c["low"], 1 + c["high"]):  # (on a border within rounding either branch would be right)
        ratio = torch.where((ratio - math.log(border)).abs() < 1e-3, ratio + 3e-3, ratio)
    return dict(logits=x, tokens=tokens, weight=weight, advantage=advantage, old=logp - ratio if c["old"] else None,
                ref=logp + torch.randn(rows, generator=g, device="cuda") * 0.4 if c["kl"] else None)


def _lengths(c):
    """Lengths of the 2 * pairs sequences: of ragged ones, spread over a quarter of the longest to all of it."""
    n, longest = 2 * c["pairs"], c["length"]
    return [max(1, longest - (i * 37 + 11) % max(1, longest * 3 // 4)) if c["ragged"] else longest for i in range(n)]


def _prepare_preference(c, g):
    lengths = _lengths(c)
    rows = sum(lengths)
    x = _matrix(c, rows, g, 3.0)
    tokens, logp = _sampled(x, 1.0, g)
    offsets = torch.tensor([0] + lengths).cumsum(0).int()
    at = torch.cat([torch.arange(n) for n in lengths])
    live = torch.tensor([max(1, n - c["prefix"]) for n in lengths]).repeat_interleave(torch.tensor(lengths))
    weight = torch.where(at < c["prefix"], 0.0, 1.0 / live if c["mean"] else 1.0).float()
    ref = logp + torch.randn(rows, generator=g, device="cuda") * 0.3 if c["reference"] else None
    return dict(logits=x, tokens=tokens, offsets=offsets.cuda(), weight=weight.cuda(), ref=ref,
                pair_weight=torch.full((c["pairs"],), 1.0 / c["pairs"], device="cuda"))


def _shapes(c):
    D, F, V = c["dim"], c["ffn"], c["vocab"]
    layer = [(D,), (3 * D, D), (D, D), (D,), (2 * F, D), (D, F)]
    return [(V, D)] + layer * c["layers"] + [(D,), (V, D)]


def _types(c):
    """Types of the gradients: of mixed ones, the gains of the norms stay in fp32."""
    return ["fp32" if c["dtype"] == "fp32" or c["dtype"] == "mixed" and len(s) == 1 else "bf16" for s in _shapes(c)]


def _flat(c):
    """Gradients as views of one buffer a type, as bucketed gradients and an optimizer's buffers are: (buffers, views)."""
    places, ends = [], {"fp32": 0, "bf16": 0}
    for shape, kind in zip(_shapes(c), _types(c)):
        places.append((kind, ends[kind], shape))
        ends[kind] += -(-math.prod(shape) // c["align"]) * c["align"]
    flat = {kind: torch.zeros(n, dtype=_T[kind], device="cuda") for kind, n in ends.items() if n}
    return list(flat.values()), [flat[kind][at:at + math.prod(shape)].view(shape) for kind, at, shape in places]


def _prepare_clip(c, g):
    flat, gradients = _flat(c)
    for i, x in enumerate(gradients):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda").mul_(10.0 ** (-1 - i * 7 % 4)))
        if i == 0:  # rows of tokens that the batch does not have
            x[torch.rand(x.shape[0], generator=g, device="cuda") < 0.6] = 0.0
    if c["norm"] == "2":
        norm = math.sqrt(sum(float(x.float().square().sum()) for x in flat))
    else:
        norm = max(float(x.abs().max()) for x in flat)
    st = dict(flat=flat, gradients=gradients, limit=norm * (0.3 if c["clipped"] else 3.0), out=None)
    if c["clipped"]:
        st["flat_out"], st["out"] = _flat(c)
    return st


def prepare(case, seed):
    make = {"logprobs": _prepare_logprobs, "policy": _prepare_policy, "preference": _prepare_preference, "clip": _prepare_clip}
    return dict(make[case["op"]](case, _generator(seed)), case=case)


# ------------------------------------------------------------------ plain forms
def _log_softmax(x):
    y = x - x.max(-1, keepdim=True).values
    return y - torch.log(torch.exp(y).sum(-1, keepdim=True))


def _entropy_terms(logq):
    """(q, q log q), zero where there is no mass."""
    q = torch.exp(logq)
    return q, torch.where(q > 0, q * logq, 0.0)


def _token_gradient(q, tokens, a):
    """a (1[v = token] - q_v)"""
    g = -q * a[:, None]
    return g.scatter_add_(1, tokens[:, None], a[:, None])


def _plain_logprobs(st):
    c = st["case"]
    tokens = st["tokens"].long()
    logq = _log_softmax(st["logits"].float() / c["temperature"])
    q, qlogq = _entropy_terms(logq)
    entropy = -qlogq.sum(-1)
    if not c["backward"]:
        logp = logq.gather(1, tokens[:, None])[:, 0]
        return (logp, entropy) if c["entropy"] else (logp,)
    grad = _token_gradient(q, tokens, st["d_logp"])
    if c["entropy"]:
        grad = grad - st["d_entropy"][:, None] * (qlogq + q * entropy[:, None])
    return ((grad / c["temperature"]).to(st["logits"].dtype),)


def _plain_policy(st):
    c = st["case"]
    tokens, A, w = st["tokens"].long(), st["advantage"], st["weight"]
    logq = _log_softmax(st["logits"].float() / c["temperature"])
    logp = logq.gather(1, tokens[:, None])[:, 0]
    r = torch.exp(logp - st["old"]) if c["old"] else torch.ones_like(logp)
    kept, held = r * A, r.clamp(1 - c["low"], 1 + c["high"]) * A
    gain = torch.minimum(kept, held)
    a = torch.where(kept <= held, -kept, 0.0)
    if c["dual"]:
        floor = torch.where(A < 0, c["dual"] * A, float("-inf"))
        a = torch.where(gain < floor, 0.0, a)
        gain = torch.maximum(gain, floor)
    loss = -gain
    if c["kl"]:
        d = st["ref"] - logp
        loss = loss + c["kl"] * (torch.expm1(d) - d)
        a = a - c["kl"] * torch.expm1(d)
    q, qlogq = _entropy_terms(logq)
    if c["entropy"]:
        entropy = -qlogq.sum(-1)
        loss = loss - c["entropy"] * entropy
    live = w != 0
    out = torch.where(live, loss, 0.0), torch.where(live, logp, 0.0)
    if not c["grad"]:
        return out
    grad = _token_gradient(q, tokens, a)
    if c["entropy"]:
        grad = grad + c["entropy"] * (qlogq + q * entropy[:, None])
    return (*out, (grad * (w / c["temperature"])[:, None]).to(st["logits"].dtype))


def _sides(c, lengths):
    """Rows of the chosen and of the rejected sequence of every pair, as ranges."""
    ends = [0]
    for n in lengths:
        ends.append(ends[-1] + n)
    P = c["pairs"]
    for p in range(P):
        i, j = (2 * p, 2 * p + 1) if c["interleaved"] else (p, P + p)
        yield (ends[i], ends[i + 1], i), (ends[j], ends[j + 1], j)


def _plain_pairs(c, h):
    """(loss, d loss / d h) of every pair, in 64 bits."""
    if c["kind"] == "square":
        return (h - 0.5 / c["beta"]) ** 2, 2 * (h - 0.5 / c["beta"])
    z = c["beta"] * h - c["margin"]
    if c["kind"] == "hinge":
        return (1 - z).clamp(min=0), torch.where(z < 1, -c["beta"], 0.0)
    s = c["smoothing"]
    up = torch.log(1 + torch.exp(-z.abs()))
    loss = (1 - s) * (up + (-z).clamp(min=0)) + s * (up + z.clamp(min=0))
    return loss, c["beta"] * (1 / (1 + torch.exp(-z)) - (1 - s))


def _plain_preference(st):
    c = st["case"]
    tokens, w, P = st["tokens"].long(), st["weight"], c["pairs"]
    logq = _log_softmax(st["logits"].float())
    logp = logq.gather(1, tokens[:, None])[:, 0]
    rows = tokens.shape[0]
    seq = torch.searchsorted(st["offsets"].long(), torch.arange(rows, device="cuda"), right=True) - 1
    pair, rejected = (seq // 2, seq % 2) if c["interleaved"] else (seq % P, seq // P)
    ratio = w.double() * (logp - st["ref"] if c["reference"] else logp).double()
    sums = torch.zeros(2 * P, dtype=torch.float64, device="cuda").index_add_(0, seq, ratio)
    both = sums.view(P, 2) if c["interleaved"] else sums.view(2, P).t()
    loss, slope = _plain_pairs(c, both[:, 0] - both[:, 1])
    out = loss.float(), sums.float()
    if not c["grad"]:
        return out
    a = (slope * st["pair_weight"])[pair] * torch.where(rejected == 1, -1.0, 1.0) * w
    return (*out, _token_gradient(torch.exp(logq), tokens, a.float()).to(st["logits"].dtype))


def _plain_clip(st):
    c = st["case"]
    if c["norm"] == "2":
        norm = torch.stack([x.float().square().sum() for x in st["gradients"]]).double().sum().sqrt()
    else:
        norm = torch.stack([x.float().abs().max() for x in st["gradients"]]).max().double()
    scale = (st["limit"] / (norm + 1e-6)).clamp(max=1.0).float()
    return [norm.float()] + [(x.float() * scale).to(x.dtype) for x in st["flat"]]


# ------------------------------------------------------------------ one pass
def _own(st):
    from paper_2608_18183_b200 import binding

    c = st["case"]
    if c["op"] == "logprobs":
        if c["backward"]:
            return (binding.hbsjd_token_logprobs_grad(st["logits"], st["tokens"], st["d_logp"], st["d_entropy"],
                                                      temperature=c["temperature"]),)
        out = binding.hbsjd_token_logprobs(st["logits"], st["tokens"], temperature=c["temperature"], want_entropy=c["entropy"])
        return out if c["entropy"] else out[:1]
    if c["op"] == "policy":
        loss, grad, logp, _ = binding.hbsjd_policy_loss(
            st["logits"], st["tokens"], st["advantage"], st["old"], st["ref"], weight=st["weight"], temperature=c["temperature"],
            clip_low=c["low"], clip_high=c["high"], dual_clip=c["dual"], kl=c["kl"], entropy=c["entropy"], want_grad=c["grad"])
        return (loss, logp, grad) if c["grad"] else (loss, logp)
    if c["op"] == "preference":
        loss, grad, sums = binding.hbsjd_preference_loss(
            st["logits"], st["tokens"], st["offsets"], st["ref"], weight=st["weight"], pair_weight=st["pair_weight"], kind=c["kind"],
            beta=c["beta"], smoothing=c["smoothing"], margin=c["margin"], interleaved=c["interleaved"], want_grad=c["grad"])
        return (loss, sums, grad) if c["grad"] else (loss, sums)
    norm = binding.hbsjd_clip_gradients(st["gradients"], st["limit"], norm=c["norm"], out=st["out"])
    return [norm] + (st["flat_out"] if c["clipped"] else st["flat"])


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "policy": _plain_policy, "preference": _plain_preference,
            "clip": _plain_clip}[state["case"]["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "clip":
        n = [math.prod(s) for s in _shapes(c)]
        nbytes = sum(a * _SIZE[kind] for a, kind in zip(n, _types(c)))
        return {"bytes": nbytes * (2 if c["clipped"] else 1) + 4, "flops": sum(n) * (3 if c["clipped"] else 2)}
    V, e = c["vocab"], _SIZE[c["dtype"]]
    if c["op"] == "logprobs":
        out = c["rows"] * (V * e + 4 + 4 * c["entropy"]) if c["backward"] else c["rows"] * (4 + 4 * c["entropy"])
        return {"bytes": c["rows"] * (V * e + 4) + out, "flops": c["rows"] * V * (4 + 2 * c["entropy"] + 3 * c["backward"])}
    if c["op"] == "policy":
        live = c["rows"] - _left_out(c)
        nbytes = live * (V * e + 8 + 4 * c["old"] + 4 * (c["kl"] > 0)) + c["rows"] * (12 + c["grad"] * V * e)
        return {"bytes": nbytes, "flops": live * V * (4 + 2 * (c["entropy"] > 0) + 3 * c["grad"])}
    lengths = _lengths(c)
    rows, live = sum(lengths), sum(max(0, n - c["prefix"]) for n in lengths)
    nbytes = live * (V * e + 4 + 4 * c["reference"]) + rows * (4 + c["grad"] * V * e) + c["pairs"] * 24
    return {"bytes": nbytes, "flops": live * V * (4 + 3 * c["grad"])}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_row_gradient(x, tokens, a, b, tau):
    """d (a logp + b entropy) / d logits."""
    q = torch.softmax(x.double() / tau, -1)
    hot = torch.nn.functional.one_hot(tokens.long(), x.shape[1])
    logq = torch.log_softmax(x.double() / tau, -1)
    grad = a[:, None] * (hot - q)
    if b is not None:
        surprise = torch.where(q > 0, -logq, 0.0)
        mean = (q * surprise).sum(-1, keepdim=True)
        grad = grad + b[:, None] * q * (surprise - mean)
    return grad / tau


def _exact_rows(x, tokens, tau):
    """(log-probability, entropy) of every row."""
    logp, entropy = [], []
    for part, t in zip(x.split(1024), tokens.split(1024)):
        d = torch.distributions.Categorical(logits=part.double() / tau)
        logp.append(d.log_prob(t.long()))
        q = d.probs
        entropy.append(-torch.special.xlogy(q, q).sum(-1))
    return torch.cat(logp), torch.cat(entropy)


def _exact_gradient(x, tokens, a, b, tau):
    parts = range(0, x.shape[0], 1024)
    return torch.cat([_exact_row_gradient(x[r:r + 1024], tokens[r:r + 1024], a[r:r + 1024], None if b is None else b[r:r + 1024], tau)
                      for r in parts])


def _exact_policy(c, st):
    logp, entropy = _exact_rows(st["logits"], st["tokens"], c["temperature"])
    at = logp.clone().requires_grad_()
    A = st["advantage"].double()
    ratio = (at - (st["old"].double() if c["old"] else logp)).exp()
    gain = torch.min(ratio * A, torch.clip(ratio, 1 - c["low"], 1 + c["high"]) * A)
    if c["dual"]:
        gain = torch.where(A < 0, torch.max(gain, c["dual"] * A), gain)
    loss = -gain
    if c["kl"]:
        d = st["ref"].double() - at
        loss = loss + c["kl"] * (d.exp() - 1 - d)
    slope, = torch.autograd.grad(loss.sum(), at)
    loss = loss.detach() - c["entropy"] * entropy
    w = st["weight"].double()
    out = torch.where(w != 0, loss, 0.0), torch.where(w != 0, logp, 0.0)
    if not c["grad"]:
        return out
    b = -c["entropy"] * w if c["entropy"] else None
    return (*out, _exact_gradient(st["logits"], st["tokens"], slope * w, b, c["temperature"]))


def _exact_preference(c, st):
    logp, _ = _exact_rows(st["logits"], st["tokens"], 1.0)
    leaf = logp.clone().requires_grad_()
    terms = st["weight"].double() * (leaf - st["ref"].double() if c["reference"] else leaf)
    sums, losses = [None] * (2 * c["pairs"]), []
    for (i0, i1, i), (j0, j1, j) in _sides(c, _lengths(c)):
        sums[i], sums[j] = terms[i0:i1].sum(), terms[j0:j1].sum()
        h = sums[i] - sums[j]
        if c["kind"] == "square":
            losses.append((h - 1 / (2 * c["beta"])).square())
        elif c["kind"] == "hinge":
            losses.append(torch.relu(1 - (c["beta"] * h - c["margin"])))
        else:
            z, F = c["beta"] * h - c["margin"], torch.nn.functional.logsigmoid
            losses.append(-(1 - c["smoothing"]) * F(z) - c["smoothing"] * F(-z))
    loss = torch.stack(losses)
    out = loss.detach(), torch.stack(sums).detach()
    if not c["grad"]:
        return out
    slope, = torch.autograd.grad((loss * st["pair_weight"].double()).sum(), leaf)
    return (*out, _exact_gradient(st["logits"], st["tokens"], slope, None, 1.0))


def exact(case, seed):
    """What `run` returns for these inputs by the operators' definitions in 64 bits."""
    c, st = case, prepare(case, seed)
    if c["op"] == "policy":
        return _exact_policy(c, st)
    if c["op"] == "preference":
        return _exact_preference(c, st)
    if c["op"] == "logprobs":
        if c["backward"]:
            b = st["d_entropy"].double() if c["entropy"] else None
            return (_exact_gradient(st["logits"], st["tokens"], st["d_logp"].double(), b, c["temperature"]),)
        out = _exact_rows(st["logits"], st["tokens"], c["temperature"])
        return out if c["entropy"] else out[:1]
    flat = [x.double() for x in st["flat"]]
    norm = math.sqrt(sum(float(torch.dot(x, x)) for x in flat)) if c["norm"] == "2" else max(float(x.abs().max()) for x in flat)
    scale = min(1.0, st["limit"] / (norm + 1e-6))
    return [torch.tensor(norm, dtype=torch.float64)] + [x * scale for x in flat]
