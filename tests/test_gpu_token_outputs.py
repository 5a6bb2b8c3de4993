"""Outputs that may be left out: every one alone, through the C entries, has the bits that it has beside the others; and the log-probabilities that
hbsjd_preference_loss gives out."""
import ctypes as C

import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _gen, _rows
from tests.token_reference import HALF, Rows, near, sampled

pytestmark = pytest.mark.gpu

# few rows (parts of clusters), many short ones, many that a CTA takes tile by tile
SHAPES = [(24, 16384, "fp32"), (700, 1001, "bf16"), (300, 49409, "fp32"), (300, 49409, "bf16")]


def _inputs(rows, V, dtype):
    import torch
    x, g = _rows(V, rows, V, 3.0, dtype, 0, 1), _gen(rows)
    t = sampled(x, 1.0, g)
    t[3] = -1
    w = torch.rand(rows, generator=g, device="cuda")
    w[5] = 0.0
    ref = torch.randn(rows, generator=g, device="cuda") - 8
    return x, t, w, ref, torch.randn(rows, generator=g, device="cuda")


def _alone(entry, desc, inputs, outs, wanted):
    """The entry with one of its outputs (pointers in order; the others NULL), which starts as what nothing writes."""
    import torch
    out = torch.full_like(outs[wanted], 77.0)
    ptr = [out.data_ptr() if i == wanted else None for i in range(len(outs))]
    rc = entry(torch.cuda.current_stream().cuda_stream, C.byref(desc), *[None if x is None else x.data_ptr() for x in inputs], *ptr)
    assert rc == 0, binding.load().hbsjd_last_error(None)
    return out


@pytest.mark.parametrize("rows,V,dtype", SHAPES)
def test_one_output_at_a_time(rows, V, dtype):
    import torch
    L = binding.load()
    x, t, w, ref, A = _inputs(rows, V, dtype)
    kind = binding.DTYPE_FP32 if dtype == "fp32" else binding.DTYPE_BF16
    d = binding.hbsjd_token_desc(rows, V, kind, 0, V, 0, 1.0, 0)
    want = binding.hbsjd_token_logprobs(x, t)
    assert torch.equal(_alone(L.hbsjd_token_logprobs, d, (x, t), want, 1), want[1])
    assert torch.equal(_alone(L.hbsjd_token_logprobs, d, (x, t), want, 0), binding.hbsjd_token_logprobs(x, t, want_entropy=False)[0])
    for bonus in (0.0, 0.01):
        p = binding.hbsjd_policy_desc(rows, V, kind, 0, V, V, 1.0, 0.2, 0.2, 0.0, 0.1, bonus)
        loss, grad, logp, _ = binding.hbsjd_policy_loss(x, t, A, ref, ref, w, kl=0.1, entropy=bonus)
        H = binding.hbsjd_policy_loss(x, t, A, ref, ref, w, kl=0.1, entropy=bonus, want_grad=False, want_entropy=True)[3]
        outs = (loss, logp, H, grad)
        for i in range(4):
            assert torch.equal(_alone(L.hbsjd_policy_loss, p, (x, t, A, ref, ref, w), outs, i), outs[i]), i
    q = binding.hbsjd_preference_desc(rows, V, kind, 2, 0, 0, V, V, 1.0, 0.1, 0.0, 0.0)
    offsets = torch.tensor([0, 7, 12, 12, rows], device="cuda").int()
    work = torch.empty(L.hbsjd_preference_workspace(q), dtype=torch.uint8, device="cuda")
    loss, grad, sums, logp = binding.hbsjd_preference_loss(x, t, offsets, ref, w, want_logp=True)
    outs = (loss, sums, logp, grad)
    for i in range(4):
        assert torch.equal(_alone(L.hbsjd_preference_loss, q, (x, t, offsets, ref, w, None, work), outs, i), outs[i]), i


@pytest.mark.parametrize("rows,V,dtype", SHAPES)
def test_log_probabilities_beside_a_preference_loss(rows, V, dtype):
    import torch
    x, t, w, ref, _ = _inputs(rows, V, dtype)
    offsets = torch.tensor([0, 9, rows - 2], device="cuda").int()
    plain = binding.hbsjd_preference_loss(x, t, offsets, ref, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for got in (binding.hbsjd_preference_loss(x, t, offsets, ref, w, want_logp=True),
                binding.hbsjd_preference_loss(x, t, offsets, ref, w, want_logp=True, stream=side)):
        torch.cuda.current_stream().wait_stream(side)
        assert len(got) == 4 and all(torch.equal(a, b) for a, b in zip(got, plain))
        r = Rows(x, t, 1.0)
        left = ~r.live | (w == 0)
        near(got[3], torch.where(left, 0.0, r.l), torch.where(left, 0.0, r.dl), HALF["fp32"])
