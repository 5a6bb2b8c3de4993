"""What hbsjd_score and hbsjd_score_topk of the binding ask of their tensors, before the library sees a pointer.  No GPU is needed: tensors are
stood in for by their attributes."""
import pytest
import torch

from paper_2608_18183_b200 import binding, synth


class _Tensor:
    is_cuda, dtype, device = True, torch.int32, torch.device("cuda", 0)

    def __init__(self, *shape, **other):
        self.shape, self.contiguous = torch.Size(shape), other.pop("contiguous", True)
        self.__dict__.update(other)

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 0x10000000


class _Library:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def _context():
    c = object.__new__(binding.Context)
    c._torch, c.shape, c.lib, c.h = torch, synth.WORKLOADS["tiny"].shape, _Library(), None
    return c


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("wrong", [dict(is_cuda=False, device=torch.device("cpu")), dict(dtype=torch.int64), dict(contiguous=False),
                                   dict(device=torch.device("cuda", 1)), dict(short=True)])
def test_score_topk_refuses(which, wrong):
    c, B = _context(), 4
    shapes = [(B, c.shape.T), (B,), (B,)]
    wrong = dict(wrong)
    if wrong.pop("short", False):
        shapes[which] = (*shapes[which][:-1], shapes[which][-1] - 1)
    if which == 0 and "device" in wrong and wrong.get("is_cuda", True):
        pytest.skip("the others are compared with the tokens' device")
    args = [_Tensor(*s) for s in shapes]
    args[which] = _Tensor(*shapes[which], **wrong)
    with pytest.raises(AssertionError) as e:
        c.hbsjd_score_topk(*args, k=3)
    assert "was called" not in str(e.value)
