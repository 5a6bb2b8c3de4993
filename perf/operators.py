"""The distillation step's operators on rows of logits, as measurable cases through the public entry points.

What a visual on-policy distillation loop does with logits next to sampling from them:

  adjust        hbsjd_adjust_logits: guidance, penalties for repeated tokens, a bias and masks of allowed tokens on the
                logits of a round's windows, in front of hbsjd_probs / hbsjd_verify.
  topk          hbsjd_topk_logits: a teacher's K largest logits per position and the log mass of all others.
  distill_topk  hbsjd_distill_topk: the divergence of the student from those K + 1 buckets and its gradient.
  distill       hbsjd_distill: the divergence of two whole rows (the bidirectional KL of the score) and its gradient.

Sizes: the vocabulary of 16384 image tokens, windows of 32 and batches of 128 images are the library's own L workload;
vocabularies of 1000 to 65537 entries stand for other tokenizers, odd ones for rows that are not aligned.
"""
from __future__ import annotations

import math

import torch

own = False

_T = {"fp32": torch.float32, "bf16": torch.bfloat16}
_POSITIONS = 256  # positions of an image: rows are (image, position) pairs


# ------------------------------------------------------------------ cases
def _adjust(rows, vocab, dtype, guidance, window, history, masks, bias, penalties, pad):
    return dict(op="adjust", rows=rows, vocab=vocab, dtype=dtype, guidance=guidance, window=window, history=history,
                masks=masks, bias=bias, penalties=penalties, pad=pad)


def _topk(rows, vocab, dtype, k, temperature, masked, pad):
    return dict(op="topk", rows=rows, vocab=vocab, dtype=dtype, k=k, temperature=temperature, masked=masked, pad=pad)


def _distill_topk(rows, vocab, dtype, k, temperature, forward, reverse, rest, grad, prefix, pad):
    return dict(op="distill_topk", rows=rows, vocab=vocab, dtype=dtype, k=k, temperature=temperature, forward=forward,
                reverse=reverse, rest=rest, grad=grad, prefix=prefix, pad=pad)


def _distill(rows, vocab, dtype, teacher, temperature, forward, reverse, grad, prefix, pad):
    return dict(op="distill", rows=rows, vocab=vocab, dtype=dtype, teacher=teacher, temperature=temperature,
                forward=forward, reverse=reverse, grad=grad, prefix=prefix, pad=pad)


def listed():
    return [
        # eight images decoded token by token: a penalty on repeated tokens and one mask per class of images
        dict(name="adjust_few", **_adjust(8, 16384, "fp32", False, 1, 200, 4, False, True, 0)),
        # a whole round of 128 images with windows of 32, guided, every rule on
        dict(name="adjust_round", **_adjust(4096, 16384, "fp32", True, 32, 256, 8, True, True, 0)),
        # a vocabulary of text and images in bf16 whose rows are not aligned, long histories
        dict(name="adjust_odd_bf16", **_adjust(771, 50021, "bf16", False, 3, 4096, 2, True, True, 0)),
        # the teacher's distribution for the few positions of one image's window
        dict(name="topk_few", **_topk(24, 16384, "fp32", 64, 1.0, False, 0)),
        # a batch's positions
        dict(name="topk_batch", **_topk(8192, 16384, "fp32", 64, 1.0, False, 0)),
        # many entries of a wide bf16 vocabulary, a tenth of it masked
        dict(name="topk_wide_bf16", **_topk(2048, 32768, "bf16", 256, 2.0, True, 0)),
        # a few positions, forward KL alone, teacher renormalised over its entries
        dict(name="distill_topk_few", **_distill_topk(37, 16384, "fp32", 32, 1.0, 1.0, 0.0, False, True, 0, 0)),
        # a batch's positions, both directions; the first 32 positions of every image are its real prefix
        dict(name="distill_topk_batch", **_distill_topk(16384, 16384, "fp32", 64, 1.0, 0.5, 0.5, True, True, 32, 0)),
        # unaligned bf16 rows, softened
        dict(name="distill_topk_odd_bf16", **_distill_topk(3001, 24001, "bf16", 128, 2.0, 1.0, 0.0, True, True, 0, 0)),
        # the loss of Eq. 3 and its gradient: a few positions, a batch's, and both models in bf16
        dict(name="distill_few", **_distill(16, 16384, "fp32", "fp32", 1.0, 0.5, 0.5, True, 0, 0)),
        dict(name="distill_batch", **_distill(8192, 16384, "fp32", "fp32", 1.0, 0.5, 0.5, True, 32, 0)),
        dict(name="distill_bf16", **_distill(8192, 16384, "bf16", "bf16", 1.0, 0.5, 0.5, True, 0, 0)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["adjust", "topk", "distill_topk", "distill"])
    vocab = rng.choice([16384, 16384, _log_int(rng, 1000, 65537), _log_int(rng, 1000, 65537)])
    dtype = rng.choice(["fp32", "bf16"])
    pad = rng.choice([0, 0, 0, 1, 64])  # rows of a wider buffer
    cap = 8192 * 16384 // 2             # elements of a drawn case, at most
    rows = _log_int(rng, 1, max(2, min(16384, cap // vocab)))
    temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
    if op == "adjust":
        return _adjust(rows, vocab, dtype, rng.random() < 0.4, rng.choice([1, 3, 16, 32]), _log_int(rng, 1, 4096),
                       rng.choice([0, 1, 5]), rng.random() < 0.5, rng.random() < 0.7, pad)
    if op == "topk":
        return _topk(rows, vocab, dtype, _log_int(rng, 1, 512), temperature, rng.random() < 0.3, pad)
    forward, reverse = rng.choice([(1.0, 0.0), (0.0, 1.0), (0.5, 0.5), (0.9, 0.3)])
    grad, prefix = rng.random() < 0.75, min(rng.choice([0, 0, 17, 64]), rows // 2)
    if op == "distill_topk":
        return _distill_topk(rows, vocab, dtype, _log_int(rng, 1, 512), temperature, forward, reverse,
                             reverse > 0 or rng.random() < 0.6, grad, prefix, pad)
    return _distill(rows, vocab, dtype, rng.choice(["fp32", "bf16"]), temperature, forward, reverse, grad, prefix, pad)


# ------------------------------------------------------------------ inputs
def _rows(c, g, scale, dtype):
    """[rows, vocab] logits, a view of wider rows where the case has padding."""
    buf = torch.randn(c["rows"], c["vocab"] + c["pad"], generator=g, device="cuda")
    return buf.mul_(scale).to(_T[dtype])[:, :c["vocab"]]


def _left_out(c):
    return c["rows"] // _POSITIONS * c["prefix"] + min(c["rows"] % _POSITIONS, c["prefix"])


def _weight(c):
    """Weight of each position in the mean over the generated ones; 0 on the real prefix, which is left out."""
    at = torch.arange(c["rows"], device="cuda") % _POSITIONS
    return torch.where(at < c["prefix"], 0.0, 1.0 / max(1, c["rows"] - _left_out(c))).float()


def _prepare_adjust(c, g):
    rows, V, L, W = c["rows"], c["vocab"], c["history"], c["window"]
    images = -(-rows // W)
    row = torch.arange(rows, device="cuda")
    st = dict(logits=_rows(c, g, 3.5, c["dtype"]), logits_u=None, cfg_scale=1.0, bias=None, mask=None, mask_row=None,
              history=None, history_row=None, history_len=None, repetition=1.0, frequency=0.0, presence=0.0)
    if c["guidance"]:
        st["logits_u"] = _rows(c, g, 3.0, c["dtype"])
        st["cfg_scale"] = 4.0
    if c["bias"]:
        st["bias"] = torch.randn(V, generator=g, device="cuda") * 0.5
    if c["masks"]:
        # bit v & 31 of word v >> 5: token v is allowed; four tokens of five are
        words = (V + 31) // 32
        bits = torch.rand(c["masks"], words, 32, generator=g, device="cuda") < 0.8
        value = (bits.long() << torch.arange(32, device="cuda")).sum(-1)
        st["mask"] = torch.where(value >= 2 ** 31, value - 2 ** 32, value).to(torch.int32)
        # images of one class share a mask, some have none
        pick = torch.randint(-1, c["masks"], (images,), generator=g, device="cuda", dtype=torch.int32)
        st["mask_row"] = pick[row // W].contiguous()
    if c["penalties"]:
        # tokens of an image come back: a third of them are drawn from a few
        tok = torch.randint(0, V, (images, L), generator=g, device="cuda", dtype=torch.int32)
        often = torch.rand(images, L, generator=g, device="cuda") < 0.33
        st["history"] = torch.where(often, tok % min(V, 37), tok)
        # position j of an image's window sees the committed tokens and the j drafts in front of it
        cursor = torch.randint(0, max(L - W, 0) + 1, (images,), generator=g, device="cuda")
        st["history_row"] = (row // W).int()
        st["history_len"] = (cursor[row // W] + row % W).clamp(max=L).int()
        st.update(repetition=1.2, frequency=0.15, presence=0.3)
    return st


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=c)
    if c["op"] == "adjust":
        st.update(_prepare_adjust(c, g))
    elif c["op"] == "topk":
        x = _rows(c, g, 3.5, c["dtype"])
        if c["masked"]:
            x[:, torch.rand(c["vocab"], generator=g, device="cuda") < 0.1] = float("-inf")
        st["logits"] = x
    else:
        s = _rows(c, g, 3.0, c["dtype"])
        st.update(logits_s=s, weight=_weight(c))
        if c["op"] == "distill":
            t = _rows(c, g, 2.0, c["teacher"])
            st["logits_t"] = t.add_((0.6 * s).to(t.dtype))
        else:
            # the teacher's K largest of a row that agrees with the student in part
            V, K = c["vocab"], min(c["k"], c["vocab"])
            values, index, rest = [], [], []
            for part in s.split(1024):
                t = 0.6 * part.float() + torch.randn(part.shape, generator=g, device="cuda") * 2.0
                v, i = torch.topk(t, K, dim=-1)
                values.append(v)
                index.append(i.int())
                rest.append(torch.logsumexp(t.scatter(1, i, float("-inf")) / c["temperature"], -1))
            st.update(values=torch.cat(values), indices=torch.cat(index),
                      rest=torch.cat(rest) if c["rest"] else None)
    return st


# ------------------------------------------------------------------ plain forms
def _plain_adjust(st):
    x = st["logits"].float()
    rows, V = x.shape
    if st["logits_u"] is not None:
        u = st["logits_u"].float()
        x = u + st["cfg_scale"] * (x - u)
    if st["history"] is not None:
        tok = st["history"][st["history_row"].long()].long()
        seen = torch.arange(tok.shape[1], device=x.device) < st["history_len"][:, None]
        n = torch.zeros(rows, V, device=x.device).scatter_add_(1, tok, seen.float())
        pen = torch.where(x > 0, x / st["repetition"], x * st["repetition"]) - n * st["frequency"] - st["presence"]
        x = torch.where(n > 0, pen, x)
    if st["bias"] is not None:
        x = x + st["bias"]
    if st["mask"] is not None:
        v = torch.arange(V, device=x.device)
        allowed = ((st["mask"][:, v >> 5] >> (v & 31)) & 1).bool()
        hide = ~allowed[st["mask_row"].long().clamp(min=0)] & (st["mask_row"] >= 0)[:, None]
        x = torch.where(hide, float("-inf"), x)
    x = torch.where(torch.isnan(x), float("-inf"), x)
    return x.to(st["logits"].dtype)


def _log_sum_exp(x):
    m = x.max(-1, keepdim=True).values
    m = torch.where(torch.isinf(m), 0.0, m)
    return torch.log(torch.exp(x - m).sum(-1, keepdim=True)) + m


def _plain_topk(st):
    c = st["case"]
    x = st["logits"].float()
    V, k = c["vocab"], min(c["k"], c["vocab"])
    # one whole number per entry: the value's order, then the lower index first
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(V, device=x.device))
    index = (2 ** 32 - 1 - (torch.topk(key, k, dim=-1).values & (2 ** 32 - 1)))
    values = x.gather(1, index)
    rest = _log_sum_exp(x.scatter(1, index, float("-inf")) / c["temperature"])[:, 0]
    index = torch.where(torch.isinf(values), -1, index)
    return values, index.int(), rest


def _plain_distill_topk(st):
    c = st["case"]
    a, b, tau = c["forward"], c["reverse"], c["temperature"]
    x = st["logits_s"].float() / tau
    idx = st["indices"].long()
    y = st["values"] / tau
    w = st["weight"][:, None]
    if st["rest"] is not None:
        y = torch.cat([y, st["rest"][:, None]], 1)
    logp = y - _log_sum_exp(y)
    lse = _log_sum_exp(x)
    logq = x.gather(1, idx) - lse
    others = x.scatter(1, idx, float("-inf"))
    logqr = _log_sum_exp(others) - lse
    if st["rest"] is not None:
        logq = torch.cat([logq, logqr], 1)
    p, q, ratio = torch.exp(logp), torch.exp(logq), logq - logp
    fkl = (-p * ratio).sum(-1, keepdim=True)
    rkl = (q * ratio).sum(-1, keepdim=True) if b else torch.zeros_like(fkl)
    loss = torch.where(w == 0, 0.0, a * fkl + b * rkl)[:, 0]
    if not c["grad"]:
        return (loss,)
    bucket = a * (q - p)
    if b:
        bucket = bucket + b * q * (ratio - rkl)
    qv = torch.exp(others - lse)
    if st["rest"] is not None:
        grad = qv * (bucket[:, -1:] / q[:, -1:])
        bucket = bucket[:, :-1]
    else:
        grad = qv * a
    grad = grad.scatter(1, idx, bucket) * (w / tau)
    return loss, grad.to(st["logits_s"].dtype)


def _plain_distill(st):
    c = st["case"]
    a, b, tau = c["forward"], c["reverse"], c["temperature"]
    x, y = st["logits_s"].float() / tau, st["logits_t"].float() / tau
    w = st["weight"][:, None]
    logq, logp = x - _log_sum_exp(x), y - _log_sum_exp(y)
    p, q, ratio = torch.exp(logp), torch.exp(logq), logq - logp
    fkl = (-p * ratio).sum(-1, keepdim=True)
    rkl = (q * ratio).sum(-1, keepdim=True)
    loss = torch.where(w == 0, 0.0, a * fkl + b * rkl)[:, 0]
    if not c["grad"]:
        return (loss,)
    grad = (a * (q - p) + b * q * (ratio - rkl)) * (w / tau)
    return loss, grad.to(st["logits_s"].dtype)


# ------------------------------------------------------------------ one pass
def _own(st):
    from paper_2608_18183_b200 import binding

    c = st["case"]
    if c["op"] == "adjust":
        names = ("logits_u", "cfg_scale", "bias", "mask", "mask_row", "history", "history_row", "history_len",
                 "repetition", "frequency", "presence")
        return binding.hbsjd_adjust_logits(st["logits"], **{n: st[n] for n in names})
    if c["op"] == "topk":
        return binding.hbsjd_topk_logits(st["logits"], min(c["k"], c["vocab"]), temperature=c["temperature"])
    how = dict(weight=st["weight"], temperature=c["temperature"], forward=c["forward"], reverse=c["reverse"],
               want_grad=c["grad"])
    if c["op"] == "distill_topk":
        out = binding.hbsjd_distill_topk(st["logits_s"], st["values"], st["indices"], st["rest"], **how)
    else:
        out = binding.hbsjd_distill(st["logits_s"], st["logits_t"], **how)
    return out if c["grad"] else out[:1]


def run(state):
    if own:
        return _own(state)
    return {"adjust": _plain_adjust, "topk": _plain_topk, "distill_topk": _plain_distill_topk,
            "distill": _plain_distill}[state["case"]["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    size = {"fp32": 4, "bf16": 2}
    rows, V = c["rows"], c["vocab"]
    e = size[c["dtype"]]
    if c["op"] == "adjust":
        nbytes = rows * V * e * (3 if c["guidance"] else 2)
        nbytes += V * 4 * c["bias"] + c["masks"] * ((V + 31) // 32) * 4 + (rows * 4 if c["masks"] else 0)
        if c["penalties"]:
            nbytes += -(-rows // c["window"]) * c["history"] * 4 + rows * 8
        return {"bytes": nbytes, "flops": rows * V * (3 * c["guidance"] + c["bias"])}
    k = min(c.get("k", 0), V)
    if c["op"] == "topk":
        return {"bytes": rows * (V * e + k * 8 + 4), "flops": rows * V * 3}
    live = rows - _left_out(c)
    nbytes = live * V * e + rows * 8 + (rows * V * e if c["grad"] else 0)
    if c["op"] == "distill_topk":
        return {"bytes": nbytes + live * (k * 8 + (4 if c["rest"] else 0)), "flops": live * V * (6 if c["grad"] else 4)}
    return {"bytes": nbytes + live * V * size[c["teacher"]], "flops": live * V * (16 if c["grad"] else 10)}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_adjust(st):
    x = st["logits"].double()
    rows, V = x.shape
    if st["logits_u"] is not None:
        x = (1 - st["cfg_scale"]) * st["logits_u"].double() + st["cfg_scale"] * x
    if st["history"] is not None:
        L = st["history"].shape[1]
        at = torch.arange(L, device=x.device)[None, :].expand(rows, L)
        live = at < st["history_len"][:, None]
        flat = (torch.arange(rows, device=x.device)[:, None] * V + st["history"][st["history_row"].long()])[live]
        n = torch.bincount(flat, minlength=rows * V).view(rows, V)
        hit = n > 0
        rho = float(torch.tensor(st["repetition"], dtype=torch.float32))
        f, pr = (float(torch.tensor(st[k], dtype=torch.float32)) for k in ("frequency", "presence"))
        factor = torch.where(x > 0, 1.0 / rho, rho)
        x = x * torch.where(hit, factor, 1.0) - n * f - hit * pr
    if st["bias"] is not None:
        x = x + st["bias"].double()
    if st["mask"] is not None:
        words = st["mask"].long()
        bits = torch.stack([(words >> i) & 1 for i in range(32)], -1).flatten(1)[:, :V].bool()
        bits = torch.cat([bits, torch.ones_like(bits[:1])])
        x = x.masked_fill(~bits[st["mask_row"].long()], float("-inf"))
    return torch.nan_to_num(x, nan=float("-inf"), posinf=float("inf"), neginf=float("-inf"))


def _exact_topk(st):
    c = st["case"]
    k = min(c["k"], c["vocab"])
    out = [], [], []
    for part in st["logits"].split(512):
        v, i = torch.sort(part.double(), dim=-1, descending=True, stable=True)
        out[0].append(v[:, :k])
        out[1].append(torch.where(v[:, :k] == float("-inf"), -1, i[:, :k]).int())
        out[2].append(torch.logsumexp(v[:, k:] / c["temperature"], -1) if k < c["vocab"] else
                      torch.full_like(v[:, 0], float("-inf")))
    return tuple(torch.cat(o) for o in out)


def _exact_part(c, s, w, t=None, values=None, indices=None, rest=None):
    a, b, tau = c["forward"], c["reverse"], c["temperature"]
    x = s.double() / tau
    q = torch.softmax(x, -1)
    lq = torch.log_softmax(x, -1)
    if t is not None:
        lp = torch.log_softmax(t.double() / tau, -1)
        p = lp.exp()
        F, R = (p * (lp - lq)).sum(-1), (q * (lq - lp)).sum(-1)
        grad = a * (q - p) + b * q * (lq - lp - R[:, None])
    else:
        i = indices.long()
        y = values.double() / tau
        total = torch.logsumexp(y if rest is None else torch.cat([y, rest.double()[:, None]], 1), -1)
        lp = y - total[:, None]
        qk, lqk = q.gather(1, i), lq.gather(1, i)
        F = (lp.exp() * (lp - lqk)).sum(-1)
        R = torch.zeros_like(F)
        listed_ = a * (qk - lp.exp())
        scale = torch.full_like(F, a)
        if rest is not None:
            other = torch.ones_like(q).scatter_(1, i, 0.0)
            qr = (q * other).sum(-1)
            lpr = rest.double() - total
            gap = qr.log() - lpr
            F = F - lpr.exp() * gap
            R = (qk * (lqk - lp)).sum(-1) + qr * gap
            listed_ = listed_ + b * qk * (lqk - lp - R[:, None])
            scale = a * (1 - lpr.exp() / qr) + b * (gap - R)
        grad = (q * scale[:, None]).scatter(1, i, listed_)
    keep = w != 0
    loss = torch.where(keep, a * F + b * R, 0.0)
    return loss, torch.where(keep[:, None], grad * (w.double() / tau)[:, None], 0.0)


def exact(case, seed):
    """What `run` returns for these inputs by the operators' definitions in 64 bits."""
    st = prepare(case, seed)
    c = st["case"]
    if c["op"] == "adjust":
        return _exact_adjust(st)
    if c["op"] == "topk":
        return _exact_topk(st)
    loss, grad = [], []
    for r in range(0, c["rows"], 1024):
        at = slice(r, r + 1024)
        more = dict(t=st["logits_t"][at]) if c["op"] == "distill" else dict(
            values=st["values"][at], indices=st["indices"][at], rest=None if st["rest"] is None else st["rest"][at])
        l, g = _exact_part(c, st["logits_s"][at], st["weight"][at], **more)
        loss.append(l)
        if c["grad"]:
            grad.append(g)
    return (torch.cat(loss), torch.cat(grad)) if c["grad"] else (torch.cat(loss),)
