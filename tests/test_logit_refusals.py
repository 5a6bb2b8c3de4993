"""Calls that the operators on rows of logits refuse.  Nothing is launched, so made-up addresses do; no GPU is needed."""
import ctypes as C

import pytest

from paper_2608_18183_b200 import binding

A, B, D = 0x10000000, 0x20000000, 0x30000000  # addresses that no call may touch
ADJUST = dict(rows=4, V=100, dtype=0, masks=2, sequences=4, history_cap=8, ld=100, ld_u=100, ld_out=100, ld_mask=4,
              ld_history=8, cfg_scale=2.0, repetition=1.1, frequency=0.0, presence=0.0)
TOPK = dict(rows=4, V=100, dtype=0, k=5, ld=100, temperature=1.0, reserved=0)
DISTILL = dict(rows=4, V=100, dtype_s=0, dtype_t=0, k=5, reserved=0, ld_s=100, ld_t=100, ld_grad=100, temperature=1.0,
               forward=0.5, reverse=0.5, reserved2=0)
INF, NAN = float("inf"), float("nan")


def _refused(entry, desc, *pointers, code=-1):
    assert getattr(binding.load(), entry)(None, None if desc is None else C.byref(desc), *pointers) == code
    detail = binding.load().hbsjd_last_error(None)
    assert detail.startswith(entry.encode()), detail


def _adjust(change, x=A, u=None, bias=None, mask=None, mrow=None, hist=None, hrow=None, hlen=None, out=D):
    _refused("hbsjd_adjust_logits", binding.hbsjd_adjust_desc(**{**ADJUST, **change}), x, u, bias, mask, mrow, hist, hrow,
             hlen, out)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=1 << 27), dict(V=0), dict(V=131073), dict(dtype=2), dict(dtype=-1), dict(ld=-1),
    dict(ld_out=99), dict(ld_out=-100), dict(cfg_scale=INF), dict(cfg_scale=NAN), dict(repetition=0.0),
    dict(repetition=-1.0), dict(repetition=NAN), dict(repetition=INF), dict(repetition=1e-39), dict(frequency=INF),
    dict(presence=NAN)])
def test_adjust_descriptor(change):
    _adjust(change)


def test_adjust_arguments():
    _refused("hbsjd_adjust_logits", None, A, None, None, None, None, None, None, None, D)
    _adjust({}, x=None)
    _adjust({}, out=None)
    _adjust({}, x=A + 2)                                  # fp32 on two bytes
    _adjust(dict(dtype=1), out=D + 1)
    _adjust({}, bias=B + 1)
    _adjust({}, u=B + 2)
    _adjust(dict(ld_u=-1), u=B)
    _adjust(dict(masks=0), mask=B)
    _adjust(dict(ld_mask=3), mask=B)                      # 96 bits for 100 entries
    _adjust(dict(sequences=0), hist=B, hrow=B)
    _adjust(dict(history_cap=0), hist=B)
    _adjust(dict(ld_history=7), hist=B)
    _adjust(dict(sequences=3), hist=B)                    # four rows without history_row
    _adjust({}, hist=B, hlen=B + 2)
    _adjust({}, out=A + 4)                                # shifted by one entry
    _adjust({}, out=A + 400)                              # by one row
    _adjust({}, u=D + 8)
    _adjust(dict(ld=150, ld_out=150), out=A + 4 * 60)     # rows that reach into the gaps of others
    _adjust(dict(ld=150, ld_out=150), out=A - 4 * 99)


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(V=0), dict(V=1 << 20), dict(dtype=7), dict(k=0), dict(k=101), dict(k=1025, V=2000, ld=2000),
    dict(ld=-5), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF),
    dict(temperature=1e-39)])
def test_topk_descriptor(change):
    _refused("hbsjd_topk_logits", binding.hbsjd_topk_desc(**{**TOPK, **change}), A, B, D, None)


def test_topk_arguments():
    d = binding.hbsjd_topk_desc(**TOPK)
    for pointers in ((None, B, D, None), (A, None, D, None), (A, B, None, None), (A + 1, B, D, None), (A, B + 2, D, None),
                     (A, B, D, D + 3)):
        _refused("hbsjd_topk_logits", d, *pointers)
    _refused("hbsjd_topk_logits", None, A, B, D, None)


@pytest.mark.parametrize("change", [
    dict(rows=-2), dict(V=0), dict(V=131073), dict(dtype_s=3), dict(ld_s=-1), dict(ld_grad=99), dict(temperature=0.0),
    dict(temperature=NAN), dict(forward=-0.1), dict(forward=NAN), dict(reverse=INF)])
def test_distill_descriptor(change):
    d = binding.hbsjd_distill_desc(**{**DISTILL, **change})
    _refused("hbsjd_distill", d, A, B, None, D, D + (1 << 20))
    _refused("hbsjd_distill_topk", d, A, B, B, B, None, D, D + (1 << 20))


def test_distill_arguments():
    d = binding.hbsjd_distill_desc(**DISTILL)
    E = D + (1 << 20)
    for pointers in ((None, B, None, D, E), (A, None, None, D, E), (A, B, None, None, None), (A, B, B + 2, D, E),
                     (A, B, None, D + 1, E), (A, B, None, D, E + 2), (A + 2, B, None, D, E), (A, B + 1, None, D, E),
                     (A, B, None, D, A + 4), (A, B, None, D, B + 400)):
        _refused("hbsjd_distill", d, *pointers)
    for pointers in ((None, B, B, B, None, D, E), (A, None, B, B, None, D, E), (A, B, None, B, None, D, E),
                     (A, B, B, B, None, None, None), (A, B + 1, B, B, None, D, E), (A, B, B, B + 2, None, D, E),
                     (A, B, B, None, None, D, E)):        # the last: reverse without a rest
        _refused("hbsjd_distill_topk", d, *pointers)
    for k in (0, -1, 1025):
        _refused("hbsjd_distill_topk", binding.hbsjd_distill_desc(**{**DISTILL, "k": k}), A, B, B, B, None, D, E)
    _refused("hbsjd_distill", binding.hbsjd_distill_desc(**{**DISTILL, "dtype_t": 9}), A, B, None, D, E)
    _refused("hbsjd_distill", binding.hbsjd_distill_desc(**{**DISTILL, "ld_t": -3}), A, B, None, D, E)


def test_no_rows_is_nothing_to_do():
    lib = binding.load()
    assert lib.hbsjd_adjust_logits(None, C.byref(binding.hbsjd_adjust_desc(**{**ADJUST, "rows": 0})), A, None, None, None,
                                   None, None, None, None, D) == 0
    assert lib.hbsjd_topk_logits(None, C.byref(binding.hbsjd_topk_desc(**{**TOPK, "rows": 0})), A, B, D, None) == 0
    d = binding.hbsjd_distill_desc(**{**DISTILL, "rows": 0})
    assert lib.hbsjd_distill(None, C.byref(d), A, B, None, D, None) == 0
    assert lib.hbsjd_distill_topk(None, C.byref(d), A, B, B, B, None, D, None) == 0


def test_descriptor_layouts():
    # 6 int32, 5 int64, 4 float; 4 int32, int64, float, uint32; 6 int32, 3 int64, 3 float, uint32
    assert C.sizeof(binding.hbsjd_adjust_desc) == 80 and binding.hbsjd_adjust_desc.ld.offset == 24
    assert C.sizeof(binding.hbsjd_topk_desc) == 32 and binding.hbsjd_topk_desc.ld.offset == 16
    assert C.sizeof(binding.hbsjd_distill_desc) == 64 and binding.hbsjd_distill_desc.ld_s.offset == 24


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    x = torch.zeros(2, 8)
    for call in (lambda: binding.hbsjd_adjust_logits(x), lambda: binding.hbsjd_topk_logits(x, 2),
                 lambda: binding.hbsjd_distill(x, x), lambda: binding.hbsjd_distill_topk(x, x, x.int())):
        with pytest.raises(binding.HbsjdError) as e:
            call()
        assert e.value.code == -1
