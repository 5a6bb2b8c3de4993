"""Temperatures that the operators on rows of logits refuse: log2(e) / temperature has to be a number, too.  No GPU is needed."""
import ctypes as C

import pytest

from paper_2608_18183_b200 import binding
from tests.test_logit_refusals import A, B, D, DISTILL, TOPK, _refused


@pytest.mark.parametrize("temperature", [3e-39, 4e-39, 4.2e-39])
def test_inverse_is_finite_but_not_in_powers_of_two(temperature):
    t = C.c_float(temperature).value
    assert 1 / t < 3.4e38 < 1.4426950408889634 / t
    _refused("hbsjd_topk_logits", binding.hbsjd_topk_desc(**{**TOPK, "temperature": temperature}), A, B, D, None)
    d = binding.hbsjd_distill_desc(**{**DISTILL, "temperature": temperature})
    _refused("hbsjd_distill", d, A, B, None, D, D + (1 << 20))
    _refused("hbsjd_distill_topk", d, A, B, B, B, None, D, D + (1 << 20))
