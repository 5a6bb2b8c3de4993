"""Calls that the operators of training by rewards and preferences refuse.  Nothing is launched, so made-up addresses do; no GPU is
needed."""
import ctypes as C

import pytest

from paper_2608_18183_b200 import binding
from tests.test_logit_refusals import _refused

A, B, D, E = 0x10000000, 0x20000000, 0x30000000, 0x40000000  # addresses that no call may touch
INF, NAN = float("inf"), float("nan")
TOKEN = dict(rows=4, V=100, dtype=0, reserved=0, ld=100, ld_grad=100, temperature=1.0, reserved2=0)
POLICY = dict(rows=4, V=100, dtype=0, reserved=0, ld=100, ld_grad=100, temperature=1.0, clip_low=0.2, clip_high=0.2, dual_clip=0.0,
              kl=0.1, entropy=0.01)
PREF = dict(rows=4, V=100, dtype=0, pairs=2, kind=0, interleaved=0, ld=100, ld_grad=100, temperature=1.0, beta=0.1, smoothing=0.1,
            margin=0.0)
COMMON = [dict(rows=-1), dict(rows=1 << 27), dict(V=0), dict(V=131073), dict(dtype=2), dict(dtype=-1), dict(ld=-1), dict(temperature=0.0),
          dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-39)]
GRAD = [dict(ld_grad=99), dict(ld_grad=-100), dict(ld_grad=1 << 41)]


@pytest.mark.parametrize("change", COMMON)
def test_token_descriptor(change):
    d = binding.hbsjd_token_desc(**{**TOKEN, **change})
    _refused("hbsjd_token_logprobs", d, A, B, D, None)
    _refused("hbsjd_token_logprobs_grad", d, A, B, D, None, E)


@pytest.mark.parametrize("change", GRAD)
def test_gradient_rows(change):
    _refused("hbsjd_token_logprobs_grad", binding.hbsjd_token_desc(**{**TOKEN, **change}), A, B, D, None, E)
    _refused("hbsjd_policy_loss", binding.hbsjd_policy_desc(**{**POLICY, **change}), A, B, D, D, D, None, D, None, None, E)
    _refused("hbsjd_preference_loss", binding.hbsjd_preference_desc(**{**PREF, **change}), A, B, D, None, None, None, D, D, None, None, E)


def test_token_arguments():
    d = binding.hbsjd_token_desc(**TOKEN)
    for p in ((None, B, D, None), (A, None, D, None), (A, B, None, None), (A + 2, B, D, None), (A, B + 2, D, None), (A, B, D + 1, None),
              (A, B, None, D + 2)):
        _refused("hbsjd_token_logprobs", d, *p)
    for p in ((None, B, D, None, E), (A, None, D, None, E), (A, B, None, None, E), (A, B, D, None, None), (A, B, D + 1, None, E),
              (A, B, D, D + 2, E), (A, B, D, None, E + 2), (A, B, D, None, A + 4), (A, B, D, None, A + 400)):
        _refused("hbsjd_token_logprobs_grad", d, *p)
    _refused("hbsjd_token_logprobs", None, A, B, D, None)
    _refused("hbsjd_token_logprobs_grad", None, A, B, D, None, E)
    # the logits' place at another stride
    _refused("hbsjd_token_logprobs_grad", binding.hbsjd_token_desc(**{**TOKEN, "ld_grad": 120}), A, B, D, None, A)
    _refused("hbsjd_token_logprobs_grad", binding.hbsjd_token_desc(**{**TOKEN, "ld": 0}), A, B, D, None, A)


@pytest.mark.parametrize("change", COMMON + [
    dict(clip_low=-0.1), dict(clip_low=1.1), dict(clip_low=NAN), dict(clip_high=-0.1), dict(clip_high=INF), dict(clip_high=NAN),
    dict(dual_clip=1.0), dict(dual_clip=0.5), dict(dual_clip=-1.0), dict(dual_clip=NAN), dict(dual_clip=INF), dict(kl=-0.1), dict(kl=NAN),
    dict(kl=INF), dict(entropy=NAN), dict(entropy=INF)])
def test_policy_descriptor(change):
    _refused("hbsjd_policy_loss", binding.hbsjd_policy_desc(**{**POLICY, **change}), A, B, D, D, D, None, D, None, None, E)


def test_policy_arguments():
    d = binding.hbsjd_policy_desc(**POLICY)
    good = [A, B, D, D, D, D, D, D, D, E]
    for at, value in ((0, None), (1, None), (2, None), (4, None), (0, A + 1), (1, B + 1), (2, D + 1), (3, D + 2), (4, D + 3), (5, D + 1), (6, D + 1),
                      (7, D + 2), (8, D + 2), (9, E + 2), (9, A + 8)):
        p = list(good)
        p[at] = value
        _refused("hbsjd_policy_loss", d, *p)
    _refused("hbsjd_policy_loss", d, *good[:6], None, None, None, None)
    _refused("hbsjd_policy_loss", None, *good)


@pytest.mark.parametrize("change", COMMON + [
    dict(pairs=0), dict(pairs=-1), dict(pairs=1 << 27), dict(kind=3), dict(kind=-1), dict(beta=0.0), dict(beta=-1.0), dict(beta=NAN),
    dict(beta=INF), dict(smoothing=-0.1), dict(smoothing=1.1), dict(smoothing=NAN), dict(margin=NAN), dict(margin=INF), dict(kind=1), dict(kind=2),
    dict(kind=2, smoothing=0.0, margin=0.1)])
def test_preference_descriptor(change):
    _refused("hbsjd_preference_loss", binding.hbsjd_preference_desc(**{**PREF, **change}), A, B, D, None, None, None, D, D, D, None, E)


def test_preference_arguments():
    d = binding.hbsjd_preference_desc(**PREF)
    good = [A, B, D, D, D, D, D, D, D, D, E]
    for at, value in ((0, None), (1, None), (2, None), (6, None), (0, A + 1), (1, B + 1), (2, D + 1), (3, D + 2), (4, D + 3), (5, D + 1), (6, D + 8),
                      (7, D + 2), (8, D + 2), (9, D + 2), (10, E + 2), (10, A + 8)):
        p = list(good)
        p[at] = value
        _refused("hbsjd_preference_loss", d, *p)
    _refused("hbsjd_preference_loss", d, *good[:7], None, None, None, None)
    _refused("hbsjd_preference_loss", None, *good)


def _clip(change={}, gradients=(A, B), out=None, sizes=(10, 20), dtypes=(0, 1), work=D, norm=E):
    n = len(gradients)
    d = binding.hbsjd_clip_desc(**{**dict(count=n, norm=0, max_norm=1.0, reserved=0), **change})
    vp = lambda xs: None if xs is None else (C.c_void_p * n)(*xs)
    _refused("hbsjd_clip_gradients", d, vp(gradients), vp(out), (C.c_int64 * n)(*sizes), (C.c_int32 * n)(*dtypes), work, norm)


def test_clip_arguments():
    for change in (dict(count=-1), dict(count=(1 << 20) + 1), dict(norm=2), dict(norm=-1), dict(max_norm=-1.0), dict(max_norm=NAN)):
        _clip(change)
    _clip(work=None)
    _clip(norm=None)
    _clip(work=D + 8)
    _clip(norm=E + 2)
    _clip(dtypes=(0, 3))
    _clip(sizes=(-1, 4))
    _clip(sizes=(4, 1 << 41))
    _clip(gradients=(A, None))
    _clip(gradients=(A + 2, B))
    _clip(gradients=(A, B + 1))
    _clip(out=(A + 4096, B + 4097))
    _clip(gradients=(A, A))                              # twice the same
    _clip(gradients=(A, A + 36))                         # the last element
    _clip(out=(A, B + 4096))                             # one in place, one not
    _clip(out=(A + 4096, A + 4096 + 36))                 # outputs overlap
    _clip(out=(A + 4, B + 4096))                         # an output and its gradient
    _clip(out=(B + 38, B + 4096))                        # an output and another's gradient
    _refused("hbsjd_clip_gradients", None, None, None, None, None, D, E)
    one = binding.hbsjd_clip_desc(1, 0, 1.0, 0)
    _refused("hbsjd_clip_gradients", one, None, None, (C.c_int64 * 1)(4), (C.c_int32 * 1)(0), D, E)
    _refused("hbsjd_clip_gradients", one, (C.c_void_p * 1)(A), None, None, (C.c_int32 * 1)(0), D, E)
    _refused("hbsjd_clip_gradients", one, (C.c_void_p * 1)(A), None, (C.c_int64 * 1)(4), None, D, E)


def test_no_rows_is_nothing_to_do():
    lib = binding.load()
    t = binding.hbsjd_token_desc(**{**TOKEN, "rows": 0})
    assert lib.hbsjd_token_logprobs(None, C.byref(t), A, B, D, None) == 0
    assert lib.hbsjd_token_logprobs_grad(None, C.byref(t), A, B, D, None, E) == 0
    assert lib.hbsjd_policy_loss(None, C.byref(binding.hbsjd_policy_desc(**{**POLICY, "rows": 0})), A, B, D, D, D, None, D, None, None, E) == 0
    p = binding.hbsjd_preference_desc(**{**PREF, "rows": 0, "pairs": 0})
    assert lib.hbsjd_preference_loss(None, C.byref(p), A, B, D, None, None, None, D, D, None, None, E) == 0
    assert lib.hbsjd_preference_workspace(C.byref(p)) == 0 and lib.hbsjd_preference_workspace(None) == 0
    assert lib.hbsjd_clip_workspace(0) == 0 and lib.hbsjd_clip_workspace(-3) == 0 and lib.hbsjd_clip_workspace(5000) >= lib.hbsjd_clip_workspace(1) > 0


def test_descriptor_layouts():
    # 4 int32, 2 int64, float, uint32; 4 int32, 2 int64, 6 float; 6 int32, 2 int64, 4 float; 2 int32, float, uint32
    assert C.sizeof(binding.hbsjd_token_desc) == 40 and binding.hbsjd_token_desc.ld.offset == 16
    assert C.sizeof(binding.hbsjd_policy_desc) == 56 and binding.hbsjd_policy_desc.temperature.offset == 32
    assert C.sizeof(binding.hbsjd_preference_desc) == 56 and binding.hbsjd_preference_desc.ld.offset == 24
    assert C.sizeof(binding.hbsjd_clip_desc) == 16


def test_score_logprobs_without_a_context():
    assert binding.load().hbsjd_score_logprobs(None, 1, A, B, D, 1.0, E, None) == -1


def test_binding_refuses_tensors_that_are_not_on_a_gpu():
    import torch
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: binding.hbsjd_token_logprobs(x, t), lambda: binding.hbsjd_token_logprobs_grad(x, t, x[:, 0]),
                 lambda: binding.hbsjd_policy_loss(x, t, x[:, 0]), lambda: binding.hbsjd_preference_loss(x, t, t),
                 lambda: binding.hbsjd_clip_gradients([x]), lambda: binding.hbsjd_clip_gradients([]), lambda: binding.hbsjd_clip_gradients([3])):
        with pytest.raises(binding.HbsjdError) as e:
            call()
        assert e.value.code == -1
