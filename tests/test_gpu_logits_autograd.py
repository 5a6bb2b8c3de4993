"""The operators on rows of logits beside autograd: what they write in place counts as a write."""
import pytest

from paper_2608_18183_b200 import binding
from tests.test_gpu_logits import _rows

pytestmark = pytest.mark.gpu


def _calls(logits, t):
    import torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lists = binding.hbsjd_topk_logits(t, 5)
    yield lambda o: binding.hbsjd_distill(logits, t, grad=o)
    yield lambda o: binding.hbsjd_distill_topk(logits, *lists, grad=o)
    yield lambda o: binding.hbsjd_adjust_logits(logits, bias=torch.ones(logits.shape[1], device="cuda"), out=o)
    yield lambda o: binding.hbsjd_distill(logits, t, grad=o, stream=side)


def test_logits_that_a_backward_needs_may_not_be_written_over():
    import torch
    t = _rows(2, 6, 300)
    for n in range(4):
        x = _rows(1, 6, 300).requires_grad_()
        logits = x.tanh()                                       # (saves its result)
        call = list(_calls(logits.detach(), t))[n]
        before = logits._version
        call(logits.detach())
        torch.cuda.synchronize()
        assert logits._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            logits.backward(torch.ones_like(logits))


def test_gradients_in_place_where_nothing_is_saved():
    """Logits of a product: the gradient may lie in their place, and a tensor of its own gives the same."""
    import torch
    h, t = _rows(1, 6, 40), _rows(2, 6, 300)
    grads = []
    for in_place in (False, True):
        head = _rows(3, 300, 40).requires_grad_()
        logits = h @ head.t()
        before = logits._version
        _, g = binding.hbsjd_distill(logits.detach(), t, grad=logits.detach() if in_place else None)
        assert (logits._version > before) == in_place
        logits.backward(g)
        grads.append(head.grad)
    assert torch.equal(*grads)
