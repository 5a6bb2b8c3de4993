"""Thin ctypes binding of libhbsjd.so: same names as the C ABI (include/hbsjd.h), argument
marshalling only.  Every step of the rollout runs inside the CUDA library; torch supplies device
memory and the stream.  There is no fallback: a missing library or GPU raises."""
from __future__ import annotations

import array
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libhbsjd.so")

DTYPE_FP32, DTYPE_BF16 = 0, 1
VERIFY_PROB, VERIFY_GREEDY = 0, 1
EXEC_FULL, EXEC_COMPACT, EXEC_HYBRID, EXEC_SYNC = 0, 1, 2, 3
DBG_PROBS, DBG_LOGITS, DBG_SLOTS = 0, 1, 2
DBG_ACT_A, DBG_ACT_Q, DBG_ACT_O, DBG_ACT_FFN, DBG_ACT_H, DBG_KV_K, DBG_KV_V = 3, 4, 5, 6, 7, 8, 9

EXPORTS = ["hbsjd_create", "hbsjd_rollout", "hbsjd_prefill_passes", "hbsjd_rollout_host", "hbsjd_profile", "hbsjd_profile_read", "hbsjd_profile_launch_floor", "hbsjd_probs", "hbsjd_verify", "hbsjd_verify_static", "hbsjd_calibrate_gamma", "hbsjd_round", "hbsjd_tokens", "hbsjd_destroy", "hbsjd_get_state",
           "hbsjd_set_state", "hbsjd_debug_read", "hbsjd_debug_forward", "hbsjd_debug_gemm",
           "hbsjd_debug_shuffle_pages", "hbsjd_debug_fold_norm", "hbsjd_debug_fail_round",
           "hbsjd_debug_force_tile", "hbsjd_gemm", "hbsjd_bikl", "hbsjd_score", "hbsjd_strerror",
           "hbsjd_last_error", "hbsjd_adjust_logits", "hbsjd_topk_logits", "hbsjd_distill", "hbsjd_distill_topk",
           "hbsjd_score_topk", "hbsjd_token_logprobs", "hbsjd_token_logprobs_grad", "hbsjd_score_logprobs", "hbsjd_policy_loss",
           "hbsjd_preference_workspace", "hbsjd_preference_loss", "hbsjd_clip_workspace", "hbsjd_clip_gradients"]


class hbsjd_model_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("n_layers", "dim", "n_heads", "ffn_hidden", "vocab", "grid_h", "grid_w", "n_classes", "dtype")] + [
                   ("rms_eps", C.c_float), ("rope_base", C.c_float)]


class hbsjd_params(C.Structure):
    _fields_ = [("window", C.c_int32), ("history_offset", C.c_int32), ("cfg_scale", C.c_float),
                ("temperature", C.c_float), ("top_k", C.c_int32), ("verify_mode", C.c_int32),
                ("exec_mode", C.c_int32), ("gamma", C.c_int32), ("seed", C.c_uint64), ("max_rounds", C.c_int32),
                ("reserved", C.c_int32)]


class hbsjd_stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in
                ("rounds", "image_forwards", "committed", "rejects", "full_rounds", "compact_rounds",
                 "prefill_forwards", "kernel_launches")] + [("ms_total", C.c_float), ("ms_prefill", C.c_float)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class hbsjd_kernel_profile(C.Structure):
    _fields_ = [("ms", C.c_double * 4), ("work", C.c_double * 4), ("launches", C.c_int64 * 4),
                ("dropped", C.c_int64), ("gemm_ms_by_rows", C.c_double * 4), ("gemm_work_by_rows", C.c_double * 4),
                ("gemm_launches_by_rows", C.c_int64 * 4), ("gemm_bytes_by_rows", C.c_double * 4)]


PROF_CLASSES = ("gemm", "attention", "accept", "other")
PROF_GEMM_ROW_BINS = ("rows<=512", "rows<=2048", "rows<=6144", "rows>6144")


class hbsjd_verify_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in
                ("batch", "window", "T", "V", "branches", "history_offset", "greedy", "top_k")] + [
                   ("cfg_scale", C.c_float), ("temperature", C.c_float), ("seed", C.c_uint64),
                   ("round", C.c_uint32), ("reserved", C.c_uint32)]


class hbsjd_adjust_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype", "masks", "sequences", "history_cap")] + [
        (n, C.c_int64) for n in ("ld", "ld_u", "ld_out", "ld_mask", "ld_history")] + [
            (n, C.c_float) for n in ("cfg_scale", "repetition", "frequency", "presence")]


class hbsjd_topk_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype", "k")] + [("ld", C.c_int64), ("temperature", C.c_float),
                                                                        ("reserved", C.c_uint32)]


class hbsjd_distill_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype_s", "dtype_t", "k", "reserved")] + [
        (n, C.c_int64) for n in ("ld_s", "ld_t", "ld_grad")] + [
            (n, C.c_float) for n in ("temperature", "forward", "reverse")] + [("reserved2", C.c_uint32)]


class hbsjd_token_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype", "reserved")] + [(n, C.c_int64) for n in ("ld", "ld_grad")] + [
        ("temperature", C.c_float), ("reserved2", C.c_uint32)]


class hbsjd_policy_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype", "reserved")] + [(n, C.c_int64) for n in ("ld", "ld_grad")] + [
        (n, C.c_float) for n in ("temperature", "clip_low", "clip_high", "dual_clip", "kl", "entropy")]


class hbsjd_preference_desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "V", "dtype", "pairs", "kind", "interleaved")] + [
        (n, C.c_int64) for n in ("ld", "ld_grad")] + [(n, C.c_float) for n in ("temperature", "beta", "smoothing", "margin")]


class hbsjd_clip_desc(C.Structure):
    _fields_ = [("count", C.c_int32), ("norm", C.c_int32), ("max_norm", C.c_float), ("reserved", C.c_uint32)]


class HbsjdError(RuntimeError):
    def __init__(self, code, what, detail=""):
        super().__init__(f"{what}: {code} ({detail})")
        self.code = code


_lib = None


def load():
    """Loads the library (no CUDA call is made); compiles it first if it has not been built.  Raises if that fails."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            # a fresh checkout: compile in-tree (nvcc, sm_100a); there is no other implementation to fall back to
            from . import build
            build.build()
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run paper_2608_18183_b200/build.py (nvcc, sm_100a)")
        L = C.CDLL(LIB_PATH)
        vp = C.c_void_p
        L.hbsjd_create.argtypes = [C.POINTER(vp), C.POINTER(hbsjd_model_desc), vp, C.c_size_t, C.c_int, C.c_int, vp]
        L.hbsjd_rollout.argtypes = [vp, C.c_int, vp, vp, vp, C.POINTER(hbsjd_params), vp, C.POINTER(hbsjd_stats)]
        L.hbsjd_rollout_host.argtypes = [vp, C.c_int, vp, vp, vp, C.POINTER(hbsjd_params), vp,
                                         C.POINTER(hbsjd_stats)]
        L.hbsjd_prefill_passes.argtypes = [vp, C.POINTER(C.c_int64)]
        L.hbsjd_profile.argtypes = [vp, C.c_int]
        L.hbsjd_profile_read.argtypes = [vp, C.POINTER(hbsjd_kernel_profile)]
        L.hbsjd_profile_launch_floor.argtypes = [vp, C.c_int, C.POINTER(C.c_float)]
        L.hbsjd_probs.argtypes = [vp, vp, vp, C.c_int, C.c_float, C.c_float, C.c_int, vp]
        L.hbsjd_verify.argtypes = [vp, C.POINTER(hbsjd_verify_desc)] + [vp] * 8
        L.hbsjd_verify_static.argtypes = [vp, C.POINTER(hbsjd_verify_desc)] + [vp] * 8
        L.hbsjd_calibrate_gamma.argtypes = [vp, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int),
                                            C.POINTER(C.c_float), C.POINTER(C.c_float)]
        L.hbsjd_round.argtypes = [vp, C.POINTER(C.c_int)]
        L.hbsjd_tokens.argtypes = [vp, vp]
        L.hbsjd_destroy.argtypes = [vp]
        L.hbsjd_destroy.restype = None
        L.hbsjd_get_state.argtypes = [vp, vp, vp, vp, vp, C.POINTER(C.c_int32)]
        L.hbsjd_set_state.argtypes = [vp, vp, vp, vp, vp, C.c_int32]
        L.hbsjd_debug_read.argtypes = [vp, C.c_int, C.c_int, vp, C.c_size_t]
        L.hbsjd_debug_forward.argtypes = [vp, C.c_int, C.c_int]
        L.hbsjd_gemm.argtypes = [vp, vp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_int]
        L.hbsjd_debug_gemm.argtypes = [vp, vp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_uint, C.c_int]
        L.hbsjd_debug_shuffle_pages.argtypes = [vp, C.c_uint64]
        L.hbsjd_debug_fold_norm.argtypes = [vp, C.c_int]
        L.hbsjd_debug_fail_round.argtypes = [vp, C.c_int]
        L.hbsjd_debug_force_tile.argtypes = [vp, C.c_int]
        L.hbsjd_bikl.argtypes = [vp, vp, vp, C.c_int, vp]
        L.hbsjd_score.argtypes = [vp, vp, C.c_int, vp, vp, vp, vp, vp, C.POINTER(C.c_float)]
        L.hbsjd_adjust_logits.argtypes = [vp, C.POINTER(hbsjd_adjust_desc)] + [vp] * 9
        L.hbsjd_topk_logits.argtypes = [vp, C.POINTER(hbsjd_topk_desc)] + [vp] * 4
        L.hbsjd_distill.argtypes = [vp, C.POINTER(hbsjd_distill_desc)] + [vp] * 5
        L.hbsjd_distill_topk.argtypes = [vp, C.POINTER(hbsjd_distill_desc)] + [vp] * 7
        L.hbsjd_score_topk.argtypes = [vp, C.c_int, vp, vp, vp, C.c_int, C.c_float, vp, vp, vp]
        L.hbsjd_token_logprobs.argtypes = [vp, C.POINTER(hbsjd_token_desc)] + [vp] * 4
        L.hbsjd_token_logprobs_grad.argtypes = [vp, C.POINTER(hbsjd_token_desc)] + [vp] * 5
        L.hbsjd_score_logprobs.argtypes = [vp, C.c_int, vp, vp, vp, C.c_float, vp, vp]
        L.hbsjd_policy_loss.argtypes = [vp, C.POINTER(hbsjd_policy_desc)] + [vp] * 10
        L.hbsjd_preference_workspace.argtypes = [C.POINTER(hbsjd_preference_desc)]
        L.hbsjd_preference_workspace.restype = C.c_size_t
        L.hbsjd_preference_loss.argtypes = [vp, C.POINTER(hbsjd_preference_desc)] + [vp] * 11
        L.hbsjd_clip_workspace.argtypes = [C.c_int]
        L.hbsjd_clip_workspace.restype = C.c_size_t
        L.hbsjd_clip_gradients.argtypes = [vp, C.POINTER(hbsjd_clip_desc)] + [vp] * 6
        L.hbsjd_strerror.argtypes = [C.c_int]
        L.hbsjd_strerror.restype = C.c_char_p
        L.hbsjd_last_error.argtypes = [vp]
        L.hbsjd_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def make_desc(shape) -> hbsjd_model_desc:
    return hbsjd_model_desc(shape.n_layers, shape.dim, shape.n_heads, shape.ffn_hidden, shape.vocab, shape.grid_h,
                            shape.grid_w, shape.n_classes, DTYPE_FP32 if shape.dtype == "fp32" else DTYPE_BF16,
                            shape.rms_eps, shape.rope_base)


def make_params(window, history_offset, cfg_scale=1.0, temperature=1.0, top_k=0, verify_mode=VERIFY_PROB,
                exec_mode=EXEC_HYBRID, gamma=0, seed=0, max_rounds=-1) -> hbsjd_params:
    return hbsjd_params(window, history_offset, cfg_scale, temperature, top_k, verify_mode, exec_mode, gamma, seed,
                        max_rounds, 0)


def hbsjd_verify_static(stream, desc, logits, q_prev, p_out, cursor, seq, delta, qbase, m_out):
    """The allocation-free verification step: no context, scratch inside the library image.
    `stream` is a torch.cuda.Stream; tensors are device tensors, state updated in place."""
    rc = load().hbsjd_verify_static(C.c_void_p(stream.cuda_stream), C.byref(desc), logits.data_ptr(),
                                    q_prev.data_ptr(), p_out.data_ptr(), cursor.data_ptr(), seq.data_ptr(),
                                    delta.data_ptr(), qbase.data_ptr(), m_out.data_ptr())
    if rc != 0:
        raise HbsjdError(rc, "hbsjd_verify_static", load().hbsjd_strerror(rc).decode())


# ---- operators on rows of logits (see include/hbsjd.h): functions of tensors, like the C entries without a context.
# Tensors lie on one GPU, which need not be the current one.  A call goes to `stream`, or to the current stream of the tensors'
# device; inputs made on another stream have to be ordered before it by the caller, and nothing waits for the result.

_torch = None
_types = {}


def _refuse(what, why):
    raise HbsjdError(-1, what, why)


def _rows(what, name, x, device=None, dtype=None, shape=None, written=False):
    """(pointer, row stride, type) of a matrix of logits or of another element type whose rows' elements are neighbours."""
    global _torch, _types
    if _torch is None:
        import torch
        _types = {torch.float32: DTYPE_FP32, torch.bfloat16: DTYPE_BF16}
        _torch = torch  # (last: another thread that finds it uses the types)
    if not isinstance(x, _torch.Tensor) or not x.is_cuda:
        _refuse(what, f"{name} is not a tensor on a GPU")
    if device is not None and x.device != device:
        _refuse(what, f"{name} lies on {x.device}, not on {device}")
    own = x.dtype
    if own not in _types if dtype is None else own != dtype:
        _refuse(what, f"{name} has type {own}")
    size = x.shape
    if len(size) != 2 or shape is not None and size != shape:
        _refuse(what, f"{name} has shape {tuple(size)}" + (f", not {tuple(shape)}" if shape is not None else ""))
    ld, step = x.stride()
    if step != 1 and size[1] > 1:
        _refuse(what, f"{name}: the elements of a row are not neighbours")
    if size[0] <= 1:
        ld = size[1]
    if written and ld < size[1]:
        _refuse(what, f"{name}: rows overlap")
    return x.data_ptr(), ld, _types.get(own)


def _plain(x, device, dtype):
    """Whether x is a contiguous matrix of this type on this device: what needs no look at its strides."""
    return isinstance(x, _torch.Tensor) and x.dtype == dtype and x.device == device and x.is_contiguous() and x.dim() == 2


def _vector(what, name, x, device, dtype, n):
    """Pointer of a contiguous vector, or None."""
    if x is None:
        return None
    if not isinstance(x, _torch.Tensor) or x.device != device or x.dtype != dtype or x.shape != (n,) or (
            n > 1 and x.stride(0) != 1):
        _refuse(what, f"{name} has to be contiguous, of type {dtype} and shape ({n},), on {device}")
    return x.data_ptr()


def _on(what, stream, device):
    """Runs the rest of a call on the tensors' device, with `stream` current if one is given."""
    if stream is None:
        return _torch.cuda.device(device)
    if stream.device != device:
        _refuse(what, f"stream of {stream.device}, tensors on {device}")
    return _torch.cuda.stream(stream)


def _call(what, entry, device, desc, *pointers):
    rc = entry(_torch._C._cuda_getCurrentRawStream(device.index), desc, *pointers)
    if rc != 0:
        raise HbsjdError(rc, what, load().hbsjd_last_error(None).decode())


def _elsewhere(f, what, logits, stream, args, kw):
    """f again, where its tensors' device and the stream it is to use are the current ones."""
    with _on(what, stream, logits.device):
        out = f(*args, **kw)
    if stream is not None:
        # memory that its owner gives back is not to be used again before this call has run
        for x in (*args, *kw.values()):
            if isinstance(x, _torch.Tensor):
                x.record_stream(stream)
    return out


def hbsjd_adjust_logits(logits, logits_u=None, cfg_scale=1.0, bias=None, mask=None, mask_row=None, history=None,
                        history_row=None, history_len=None, repetition=1.0, frequency=0.0, presence=0.0, out=None,
                        stream=None):
    """Guidance, penalties, bias and masks on [rows, V] logits of fp32 or bf16 -> out, a new tensor or the given one (which may
    be `logits`, unless autograd needs those for a backward).  mask: int32 or uint32 words [masks, words], history: int32 [sequences, tokens], row numbers and
    lengths int32 [rows], bias fp32 [V]."""
    what = "hbsjd_adjust_logits"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_adjust_logits, what, logits, stream,
                          (logits, logits_u, cfg_scale, bias, mask, mask_row, history, history_row, history_len, repetition,
                           frequency, presence, out), {})
    shape, i32 = logits.shape, _torch.int32
    rows, V = shape
    u, ld_u = None, 0
    if logits_u is not None:
        u, ld_u, _ = _rows(what, "logits_u", logits_u, device, logits.dtype, shape)
    words, ld_mask, masks = None, 0, 0
    if mask is not None:
        if _plain(mask, device, i32):
            words = mask.data_ptr()
            ld_mask = mask.shape[1]
        else:
            words, ld_mask, _ = _rows(what, "mask", mask, device,
                                      i32 if getattr(mask, "dtype", None) == i32 else _torch.uint32)
        masks = mask.shape[0]
        if mask.shape[1] < (V + 31) // 32:
            _refuse(what, f"mask has {mask.shape[1]} words for {V} entries")
        if masks == 0:
            words = None
        elif ld_mask < mask.shape[1]:
            _refuse(what, "mask: rows overlap")
    tok, ld_history, sequences, cap = None, 0, 0, 0
    if history is not None:
        if _plain(history, device, i32):
            tok = history.data_ptr()
            ld_history = history.shape[1]
        else:
            tok, ld_history, _ = _rows(what, "history", history, device, i32, written=True)
        sequences, cap = history.shape
        if not sequences or not cap:
            tok = None
    given = out is not None
    if given:
        o, ld_out, _ = _rows(what, "out", out, device, logits.dtype, shape, written=True)
    else:
        out = _torch.empty_like(logits, memory_format=_torch.contiguous_format)
        o, ld_out = out.data_ptr(), V
    if rows == 0:
        return out
    d = hbsjd_adjust_desc(rows, V, dtype, masks, sequences, cap, ld, ld_u, ld_out, ld_mask, ld_history, cfg_scale, repetition,
                          frequency, presence)
    _call(what, load().hbsjd_adjust_logits, device, d, x, u, _vector(what, "bias", bias, device, _torch.float32, V), words,
          _vector(what, "mask_row", mask_row, device, i32, rows), tok,
          _vector(what, "history_row", history_row, device, i32, rows),
          _vector(what, "history_len", history_len, device, i32, rows), o)
    if given:
        _torch.autograd.graph.increment_version(out)  # (autograd is to know that a saved tensor has changed)
    return out


def hbsjd_topk_logits(logits, k, temperature=1.0, want_rest=True, stream=None):
    """The k largest logits of each row of [rows, V]: (values fp32 [rows, k], indices int32 [rows, k], rest fp32 [rows] or
    None)."""
    what = "hbsjd_topk_logits"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_topk_logits, what, logits, stream, (logits, k, temperature, want_rest), {})
    rows, V = logits.shape
    if not 1 <= k <= min(V, 1024):
        _refuse(what, f"k = {k} is out of range")
    values = logits.new_empty((rows, k), dtype=_torch.float32)
    indices = _torch.empty_like(values, dtype=_torch.int32)
    rest = logits.new_empty((rows,), dtype=_torch.float32) if want_rest else None
    if rows:
        _call(what, load().hbsjd_topk_logits, device, hbsjd_topk_desc(rows, V, dtype, k, ld, temperature, 0), x,
              values.data_ptr(), indices.data_ptr(), rest.data_ptr() if want_rest else None)
    return values, indices, rest


def _distill(what, entry, logits_s, s, ld_s, dtype_s, teacher, dtype_t, ld_t, k, weight, temperature, forward, reverse,
             want_grad, grad):
    """What both forms of the divergence share: the gradient and the loss, and the call."""
    shape, device = logits_s.shape, logits_s.device
    rows, V = shape
    given = grad is not None
    if given:
        g, ld_g, _ = _rows(what, "grad", grad, device, logits_s.dtype, shape, written=True)
    elif want_grad:
        grad = _torch.empty_like(logits_s, memory_format=_torch.contiguous_format)
        g, ld_g = grad.data_ptr(), V
    else:
        g, ld_g = None, 0
    w = _vector(what, "weight", weight, device, _torch.float32, rows)
    loss = logits_s.new_empty((rows,), dtype=_torch.float32) if w is None else _torch.empty_like(weight)
    if rows:
        d = hbsjd_distill_desc(rows, V, dtype_s, dtype_t, k, 0, ld_s, ld_t, ld_g, temperature, forward, reverse, 0)
        _call(what, entry, device, d, s, *teacher, w, loss.data_ptr(), g)
        if given:
            _torch.autograd.graph.increment_version(grad)
    return loss, grad


def hbsjd_distill(logits_s, logits_t, weight=None, temperature=1.0, forward=0.5, reverse=0.5, want_grad=True, grad=None,
                  stream=None):
    """forward KL(p || q) + reverse KL(q || p) of each row of the student's [rows, V] logits (q) against the teacher's (p), and
    weight times its gradient in logits_s: (loss fp32 [rows], grad like logits_s or None).  The defaults are Eq. 3.
    grad: a tensor for the gradient, which may be logits_s, unless autograd needs those for a backward (it refuses to go on then).  In a
    training step: logits_s.backward(grad)."""
    what = "hbsjd_distill"
    s, ld_s, dtype_s = _rows(what, "logits_s", logits_s)
    device = logits_s.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_distill, what, logits_s, stream,
                          (logits_s, logits_t, weight, temperature, forward, reverse, want_grad, grad), {})
    t, ld_t, dtype_t = _rows(what, "logits_t", logits_t, device, None, logits_s.shape)
    return _distill(what, load().hbsjd_distill, logits_s, s, ld_s, dtype_s, (t,), dtype_t, ld_t, 0, weight, temperature,
                    forward, reverse, want_grad, grad)


def hbsjd_distill_topk(logits_s, values, indices, rest=None, weight=None, temperature=1.0, forward=1.0, reverse=0.0,
                       want_grad=True, grad=None, stream=None):
    """hbsjd_distill against a teacher that is given by its largest logits: values fp32 and indices int32 [rows, k], rest fp32
    [rows] (the tokens that are not listed as one outcome) or None (renormalised over the list)."""
    what = "hbsjd_distill_topk"
    s, ld_s, dtype_s = _rows(what, "logits_s", logits_s)
    device = logits_s.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_distill_topk, what, logits_s, stream,
                          (logits_s, values, indices, rest, weight, temperature, forward, reverse, want_grad, grad), {})
    rows = logits_s.shape[0]
    if not (_plain(values, device, _torch.float32) and _plain(indices, device, _torch.int32) and
            values.shape == indices.shape and values.shape[0] == rows):
        _refuse(what, f"values and indices have to be contiguous matrices of fp32 and int32 with {rows} rows on {device}")
    r = _vector(what, "rest", rest, device, _torch.float32, rows)
    return _distill(what, load().hbsjd_distill_topk, logits_s, s, ld_s, dtype_s, (values.data_ptr(), indices.data_ptr(), r),
                    0, 0, values.shape[1], weight, temperature, forward, reverse, want_grad, grad)


# ---- training by rewards and preferences (see include/hbsjd.h)

PREFERENCE = {"sigmoid": 0, "hinge": 1, "square": 2}
NORM = {"2": 0, "max": 1}


def _gradient(what, grad, want, logits):
    """(tensor, pointer, row stride) of the gradient: the given tensor, a new one, or none."""
    if grad is not None:
        return (grad, *_rows(what, "grad", grad, logits.device, logits.dtype, logits.shape, written=True)[:2])
    if not want:
        return None, None, 0
    grad = _torch.empty_like(logits, memory_format=_torch.contiguous_format)
    return grad, grad.data_ptr(), logits.shape[1]


def _tokens(what, tokens, device, rows):
    if tokens is None:
        _refuse(what, "tokens are missing")
    return _vector(what, "tokens", tokens, device, _torch.int32, rows)


def hbsjd_token_logprobs(logits, tokens, temperature=1.0, want_entropy=True, stream=None):
    """Log-probability of each row's token under softmax(logits / temperature) and the entropy of that distribution: (logp fp32
    [rows], entropy fp32 [rows] or None).  logits [rows, V] of fp32 or bf16, tokens int32 [rows]; a token outside 0..V-1 leaves its row
    out (0, 0)."""
    what = "hbsjd_token_logprobs"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_token_logprobs, what, logits, stream, (logits, tokens, temperature, want_entropy), {})
    rows, V = logits.shape
    t = _tokens(what, tokens, device, rows)
    logp = logits.new_empty((rows,), dtype=_torch.float32)
    entropy = _torch.empty_like(logp) if want_entropy else None
    if rows:
        _call(what, load().hbsjd_token_logprobs, device, hbsjd_token_desc(rows, V, dtype, 0, ld, 0, temperature, 0), x, t,
              logp.data_ptr(), entropy.data_ptr() if want_entropy else None)
    return logp, entropy


def hbsjd_token_logprobs_grad(logits, tokens, d_logp, d_entropy=None, temperature=1.0, grad=None, stream=None):
    """The backward of hbsjd_token_logprobs: from a loss's derivatives in logp and entropy (fp32 [rows]; the second may be None) its
    gradient in the logits, a new tensor or the given one (which may be `logits`, unless autograd needs those for a backward)."""
    what = "hbsjd_token_logprobs_grad"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_token_logprobs_grad, what, logits, stream, (logits, tokens, d_logp, d_entropy, temperature, grad), {})
    rows, V = logits.shape
    t, f32 = _tokens(what, tokens, device, rows), _torch.float32
    if d_logp is None:
        _refuse(what, "d_logp is missing")
    a, b = _vector(what, "d_logp", d_logp, device, f32, rows), _vector(what, "d_entropy", d_entropy, device, f32, rows)
    given = grad is not None
    grad, g, ld_g = _gradient(what, grad, True, logits)
    if rows:
        _call(what, load().hbsjd_token_logprobs_grad, device, hbsjd_token_desc(rows, V, dtype, 0, ld, ld_g, temperature, 0), x, t, a, b, g)
        if given:
            _torch.autograd.graph.increment_version(grad)
    return grad


def hbsjd_policy_loss(logits, tokens, advantage, old_logp=None, ref_logp=None, weight=None, temperature=1.0, clip_low=0.2,
                      clip_high=0.2, dual_clip=0.0, kl=0.0, entropy=0.0, want_grad=True, want_entropy=False, grad=None, stream=None):
    """The clipped policy loss of each row, with `kl` times the KL estimate e^d - 1 - d against the reference (d = ref_logp - logp) and
    less `entropy` times the entropy, and weight times its gradient in the logits: (loss fp32 [rows], grad like logits or None, logp
    fp32 [rows], entropy fp32 [rows] or None).  advantage, old_logp (None: the ratio is one), ref_logp (None where kl is 0) and weight
    (None: ones; 0 leaves a row out) fp32 [rows].  grad: as in hbsjd_distill.  In a training step: logits.backward(grad)."""
    what = "hbsjd_policy_loss"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_policy_loss, what, logits, stream,
                          (logits, tokens, advantage, old_logp, ref_logp, weight, temperature, clip_low, clip_high, dual_clip, kl, entropy,
                           want_grad, want_entropy, grad), {})
    rows, V = logits.shape
    t, f32 = _tokens(what, tokens, device, rows), _torch.float32
    if advantage is None:
        _refuse(what, "advantage is missing")
    row = [_vector(what, name, v, device, f32, rows) for name, v in (
        ("advantage", advantage), ("old_logp", old_logp), ("ref_logp", ref_logp), ("weight", weight))]
    given = grad is not None
    grad, g, ld_g = _gradient(what, grad, want_grad, logits)
    loss = logits.new_empty((rows,), dtype=f32)
    logp = _torch.empty_like(loss)
    H = _torch.empty_like(loss) if want_entropy else None
    if rows:
        d = hbsjd_policy_desc(rows, V, dtype, 0, ld, ld_g, temperature, clip_low, clip_high, dual_clip, kl, entropy)
        _call(what, load().hbsjd_policy_loss, device, d, x, t, *row, loss.data_ptr(), logp.data_ptr(),
              H.data_ptr() if want_entropy else None, g)
        if given:
            _torch.autograd.graph.increment_version(grad)
    return loss, grad, logp, H


def hbsjd_preference_loss(logits, tokens, offsets, ref_logp=None, weight=None, pair_weight=None, temperature=1.0, beta=0.1,
                          kind="sigmoid", smoothing=0.0, margin=0.0, interleaved=False, want_grad=True, grad=None, stream=None,
                          want_logp=False):
    """The loss of pairs of sequences, one preferred to the other, and its gradient in the logits: (loss fp32 [pairs], grad like
    logits or None, sums fp32 [2 pairs]: weight (logp - ref_logp) summed over each sequence), and with want_logp behind them the tokens'
    log-probabilities, fp32 [rows] (0: left out), for a likelihood term beside it.  Sequence s is rows offsets[s] ..
    offsets[s + 1] - 1 (int32 [2 pairs + 1]); the chosen ones are the even ones if interleaved, else the first half.  ref_logp, weight
    fp32 [rows], pair_weight fp32 [pairs] or None.  kind: "sigmoid", "hinge" or "square" (see include/hbsjd.h).  grad: as in
    hbsjd_distill."""
    what = "hbsjd_preference_loss"
    x, ld, dtype = _rows(what, "logits", logits)
    device = logits.device
    if stream is not None or device.index != _torch.cuda.current_device():
        return _elsewhere(hbsjd_preference_loss, what, logits, stream,
                          (logits, tokens, offsets, ref_logp, weight, pair_weight, temperature, beta, kind, smoothing, margin, interleaved,
                           want_grad, grad, None, want_logp), {})
    rows, V = logits.shape
    t, f32 = _tokens(what, tokens, device, rows), _torch.float32
    if kind not in PREFERENCE:
        _refuse(what, f"unknown loss {kind!r}")
    count = offsets.shape[0] if isinstance(offsets, _torch.Tensor) and offsets.dim() == 1 else 0
    if count < 3 or count % 2 == 0:
        _refuse(what, "offsets are to be a vector of 2 pairs + 1")
    pairs = count // 2
    at = _vector(what, "offsets", offsets, device, _torch.int32, count)
    ref, w = _vector(what, "ref_logp", ref_logp, device, f32, rows), _vector(what, "weight", weight, device, f32, rows)
    pw = _vector(what, "pair_weight", pair_weight, device, f32, pairs)
    given = grad is not None
    grad, g, ld_g = _gradient(what, grad, want_grad, logits)
    loss, sums = logits.new_empty((pairs,), dtype=f32), logits.new_empty((2 * pairs,), dtype=f32)
    logp = logits.new_empty((rows,), dtype=f32) if want_logp else None
    if not rows:
        _refuse(what, "sequences without a row")
    d = hbsjd_preference_desc(rows, V, dtype, pairs, PREFERENCE[kind], 1 if interleaved else 0, ld, ld_g, temperature, beta, smoothing,
                              margin)
    L = load()
    work = logits.new_empty((L.hbsjd_preference_workspace(d),), dtype=_torch.uint8)
    _call(what, L.hbsjd_preference_loss, device, d, x, t, at, ref, w, pw, work.data_ptr(), loss.data_ptr(), sums.data_ptr(),
          logp.data_ptr() if want_logp else None, g)
    if given:
        _torch.autograd.graph.increment_version(grad)
    return (loss, grad, sums, logp) if want_logp else (loss, grad, sums)


def _dense(x):
    """Whether x's elements fill one stretch of memory, in any order."""
    if x.is_contiguous():
        return True
    size = 1
    for step, n in sorted((s, n) for s, n in zip(x.stride(), x.shape) if n != 1):
        if step != size:
            return False
        size *= n
    return True


def hbsjd_clip_gradients(gradients, max_norm=float("inf"), norm="2", out=None, stream=None):
    """The norm of all gradients (a list of dense fp32 or bf16 tensors on one GPU) as one vector, a new fp32 scalar on that GPU; they are
    scaled in place by min(1, max_norm / (norm + 1e-6)), or into `out`, tensors like them, which get copies where nothing is scaled.
    norm: "2" or "max" (the largest magnitude).  An infinite or NaN norm scales nothing.  max_norm = inf: the norm alone.  No two
    tensors may overlap."""
    what = "hbsjd_clip_gradients"
    gradients = list(gradients)
    if not gradients:
        _refuse(what, "no gradients")
    if _torch is None:
        try:
            _rows(what, "gradients", None)  # (finds torch)
        except HbsjdError:
            pass
    outs = None if out is None else list(out)
    if norm not in NORM:
        _refuse(what, f"unknown norm {norm!r}")
    if outs is not None and len(outs) != len(gradients):
        _refuse(what, f"{len(outs)} outputs for {len(gradients)} gradients")
    # (what there are many of is looked at without a loop's words a tensor: 75 gradients 67 us in place of 39)
    T = _torch.Tensor
    try:
        index = T.get_device(gradients[0])
        if index < 0 or set(map(T.get_device, gradients)) != {index}:
            _refuse(what, "gradients have to lie on one GPU")
        types = [_types[x.dtype] for x in gradients]
        if outs is not None and (set(map(T.get_device, outs)) != {index} or [x.dtype for x in outs] != [x.dtype for x in gradients] or
                                 list(map(T.size, outs)) != list(map(T.size, gradients))):
            _refuse(what, "outputs have to be like the gradients")
        if not all(map(T.is_contiguous, gradients)) or outs is not None and not all(map(T.is_contiguous, outs)):
            for i, x in enumerate(gradients):
                if not _dense(x):
                    _refuse(what, f"gradients[{i}] is not dense")
                if outs is not None and outs[i].stride() != x.stride():
                    _refuse(what, f"out[{i}] has its elements in another order than gradients[{i}]")
    except (TypeError, KeyError, RuntimeError) as e:
        if isinstance(e, HbsjdError):
            raise
        _refuse(what, f"gradients and outputs have to be tensors of fp32 or bf16 on a GPU ({e})")
    if stream is not None or index != _torch.cuda.current_device():
        device = gradients[0].device
        with _on(what, stream, device):
            result = hbsjd_clip_gradients(gradients, max_norm, norm, outs)
        if stream is not None:
            for x in gradients + (outs or []):
                x.record_stream(stream)
        return result
    n = len(gradients)
    L = load()
    places = array.array("Q", map(T.data_ptr, gradients))
    places.extend(map(T.data_ptr, outs or ()))
    sizes, kinds = array.array("q", map(T.numel, gradients)), array.array("i", types)
    at = places.buffer_info()[0]
    result = gradients[0].new_empty((), dtype=_torch.float32)
    work = gradients[0].new_empty((L.hbsjd_clip_workspace(n),), dtype=_torch.uint8)
    _call(what, L.hbsjd_clip_gradients, result.device, hbsjd_clip_desc(n, NORM[norm], max_norm, 0), at, at + 8 * n if outs is not None else None,
          sizes.buffer_info()[0], kinds.buffer_info()[0], work.data_ptr(), result.data_ptr())
    if outs is not None or max_norm != float("inf"):
        _torch.autograd.graph.increment_version(gradients if outs is None else outs)
    return result


class Context:
    """Owner of one hbsjd_ctx.  Methods carry the names of the C entry points."""

    def __init__(self, shape, weights: np.ndarray, max_batch: int, max_window: int, stream=None):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("hbsjd needs a CUDA device; there is no CPU path")
        self._torch = torch
        self.shape = shape
        self.lib = load()
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        w = np.ascontiguousarray(weights, dtype=np.uint8)
        self.h = C.c_void_p()
        desc = make_desc(shape)
        rc = self.lib.hbsjd_create(C.byref(self.h), C.byref(desc), w.ctypes.data, w.nbytes, max_batch, max_window,
                                   C.c_void_p(self.stream.cuda_stream))
        if rc != 0:
            raise HbsjdError(rc, "hbsjd_create", self.lib.hbsjd_strerror(rc).decode())
        self.max_batch, self.max_window = max_batch, max_window
        # the library's rule for the form of RMSNorm of a bf16 context (see hbsjd_debug_fold_norm)
        self.fold_norm = shape.dtype == "bf16" and 2 * max_batch * max_window <= 2048
        self.batch = 0
        self.window = 0

    def _check(self, rc, what):
        if rc < 0:
            raise HbsjdError(rc, what, self.lib.hbsjd_last_error(self.h).decode())
        return rc

    def hbsjd_rollout(self, prefix_tokens, prefix_len, class_labels, params: hbsjd_params, out_tokens=None):
        """Device int32 tensors in, device int32 [batch, T] out.  Returns (out_tokens, stats dict)."""
        torch = self._torch
        assert prefix_tokens.is_cuda and prefix_tokens.dtype == torch.int32 and prefix_tokens.is_contiguous()
        assert prefix_len.is_cuda and prefix_len.dtype == torch.int32
        assert class_labels.is_cuda and class_labels.dtype == torch.int32
        B = prefix_tokens.shape[0]
        if out_tokens is None:
            out_tokens = torch.empty((B, self.shape.T), dtype=torch.int32, device=prefix_tokens.device)
        st = hbsjd_stats()
        rc = self.lib.hbsjd_rollout(self.h, B, prefix_tokens.data_ptr(), prefix_len.data_ptr(),
                                    class_labels.data_ptr(), C.byref(params), out_tokens.data_ptr(), C.byref(st))
        self._check(rc, "hbsjd_rollout")
        self.batch, self.window = B, params.window
        return out_tokens, st.as_dict()

    def hbsjd_rollout_host(self, prefix_tokens, prefix_len, class_labels, params: hbsjd_params, out_tokens):
        """Host int32 buffers in (numpy arrays or pinned torch CPU tensors), host int32 [batch, T] out."""
        def ptr(x):
            return x.ctypes.data if isinstance(x, np.ndarray) else x.data_ptr()
        B = prefix_tokens.shape[0]
        st = hbsjd_stats()
        rc = self.lib.hbsjd_rollout_host(self.h, B, ptr(prefix_tokens), ptr(prefix_len), ptr(class_labels),
                                         C.byref(params), ptr(out_tokens), C.byref(st))
        self._check(rc, "hbsjd_rollout_host")
        self.batch, self.window = B, params.window
        return out_tokens, st.as_dict()

    def hbsjd_prefill_passes(self) -> int:
        """Batched forwards that pre-filled the prefixes of the last rollout."""
        n = C.c_int64(0)
        self._check(self.lib.hbsjd_prefill_passes(self.h, C.byref(n)), "hbsjd_prefill_passes")
        return n.value

    def hbsjd_profile(self, enable: bool):
        self._check(self.lib.hbsjd_profile(self.h, 1 if enable else 0), "hbsjd_profile")

    def hbsjd_profile_read(self):
        p = hbsjd_kernel_profile()
        self._check(self.lib.hbsjd_profile_read(self.h, C.byref(p)), "hbsjd_profile_read")
        return {n: dict(ms=p.ms[i], work=p.work[i], launches=p.launches[i]) for i, n in enumerate(PROF_CLASSES)} | {
            "dropped": p.dropped,
            "gemm_by_rows": {n: dict(ms=p.gemm_ms_by_rows[i], work=p.gemm_work_by_rows[i],
                                     launches=p.gemm_launches_by_rows[i], bytes=p.gemm_bytes_by_rows[i])
                             for i, n in enumerate(PROF_GEMM_ROW_BINS)}}

    def hbsjd_profile_launch_floor(self, reps=200) -> float:
        """Median event bracket of an empty kernel launch, microseconds."""
        us = C.c_float(0.0)
        self._check(self.lib.hbsjd_profile_launch_floor(self.h, reps, C.byref(us)), "hbsjd_profile_launch_floor")
        return us.value

    def hbsjd_probs(self, logits_c, logits_u=None, cfg_scale=1.0, temperature=1.0, top_k=0):
        """Device fp32 [rows, V] logits -> device fp32 [rows, V] probabilities."""
        out = self._torch.empty_like(logits_c)
        self._check(self.lib.hbsjd_probs(self.h, logits_c.data_ptr(), None if logits_u is None else logits_u.data_ptr(),
                                         logits_c.shape[0], cfg_scale, temperature, top_k, out.data_ptr()),
                    "hbsjd_probs")
        return out

    def hbsjd_verify(self, desc: hbsjd_verify_desc, logits, q_prev, p_out, cursor, seq, delta, qbase, m_out):
        """Verification step on device tensors; state tensors are updated in place."""
        self._check(self.lib.hbsjd_verify(self.h, C.byref(desc), logits.data_ptr(), q_prev.data_ptr(),
                                          p_out.data_ptr(), cursor.data_ptr(), seq.data_ptr(), delta.data_ptr(),
                                          qbase.data_ptr(), m_out.data_ptr()), "hbsjd_verify")

    def hbsjd_calibrate_gamma(self, batch, window, guidance):
        """Returns (gamma, ms_full[5], ms_compact[5]) for live = batch, 3/4, 1/2, 1/4, 1/8 of the batch."""
        g = C.c_int(0)
        mf, mc = (C.c_float * 5)(), (C.c_float * 5)()
        self._check(self.lib.hbsjd_calibrate_gamma(self.h, batch, window, 1 if guidance else 0, C.byref(g), mf, mc),
                    "hbsjd_calibrate_gamma")
        self.batch = 0
        return g.value, list(mf), list(mc)

    def hbsjd_round(self) -> int:
        live = C.c_int(0)
        self._check(self.lib.hbsjd_round(self.h, C.byref(live)), "hbsjd_round")
        return live.value

    def hbsjd_tokens(self):
        out = self._torch.empty((self.batch, self.shape.T), dtype=self._torch.int32, device="cuda")
        self._check(self.lib.hbsjd_tokens(self.h, out.data_ptr()), "hbsjd_tokens")
        return out

    def hbsjd_get_state(self):
        """(round, cursor[B], seq[B,T+1], delta[B,T+1], qbase[B]) as numpy arrays."""
        B, T1 = self.batch, self.shape.T + 1
        cur = np.zeros(B, dtype=np.int32)
        seq = np.zeros((B, T1), dtype=np.int32)
        dl = np.zeros((B, T1), dtype=np.uint8)
        qb = np.zeros(B, dtype=np.int32)
        rnd = C.c_int32(0)
        self._check(self.lib.hbsjd_get_state(self.h, cur.ctypes.data, seq.ctypes.data, dl.ctypes.data,
                                             qb.ctypes.data, C.byref(rnd)), "hbsjd_get_state")
        return rnd.value, cur, seq, dl, qb

    def hbsjd_set_state(self, rnd, cursor, seq, delta, qbase):
        cur = np.ascontiguousarray(cursor, dtype=np.int32)
        seq = np.ascontiguousarray(seq, dtype=np.int32)
        dl = np.ascontiguousarray(delta, dtype=np.uint8)
        qb = np.ascontiguousarray(qbase, dtype=np.int32)
        self._check(self.lib.hbsjd_set_state(self.h, cur.ctypes.data, seq.ctypes.data, dl.ctypes.data,
                                             qb.ctypes.data, int(rnd)), "hbsjd_set_state")

    def hbsjd_debug_read(self, what, index):
        V = self.shape.vocab
        if what == DBG_SLOTS:
            buf = np.zeros((3, self.max_batch), dtype=np.int32)
            n = self._check(self.lib.hbsjd_debug_read(self.h, what, 0, buf.ctypes.data, buf.nbytes), "debug_read")
            return buf.reshape(-1)[:3 * n].reshape(3, n)
        if what >= DBG_ACT_A:
            # activation rows / cache rows in the context's element type, returned widened to fp32
            s = self.shape
            width = s.ffn_hidden if what == DBG_ACT_FFN else s.dim
            rows = s.T + 1 if what in (DBG_KV_K, DBG_KV_V) else self.window
            raw16 = s.dtype == "bf16" and what != DBG_ACT_H
            buf = np.zeros((rows, width), dtype=np.uint16 if raw16 else np.float32)
            n = self._check(self.lib.hbsjd_debug_read(self.h, what, index, buf.ctypes.data, buf.nbytes), "debug_read")
            out = buf[:n]
            return (out.astype(np.uint32) << np.uint32(16)).view(np.float32) if raw16 else out
        buf = np.zeros((self.window, V), dtype=np.float32)
        n = self._check(self.lib.hbsjd_debug_read(self.h, what, index, buf.ctypes.data, buf.nbytes), "debug_read")
        return buf[:n]

    def hbsjd_debug_forward(self, layer: int, stage: int):
        """Partial verifier forward of the current state up to `layer` (stage 0: attention sub-block, 1: whole block)."""
        self._check(self.lib.hbsjd_debug_forward(self.h, layer, stage), "hbsjd_debug_forward")

    def hbsjd_gemm(self, A, W, Cout, accumulate=False):
        """Cout[M,N] fp32 (+)= A[M,K] . W[N,K]^T, tensors of the context's element type on the GPU."""
        M, K = A.shape
        N = W.shape[0]
        assert W.shape[1] == K and tuple(Cout.shape) == (M, N) and Cout.dtype == self._torch.float32
        assert A.is_contiguous() and W.is_contiguous() and Cout.is_contiguous()
        self._check(self.lib.hbsjd_gemm(self.h, A.data_ptr(), W.data_ptr(), Cout.data_ptr(), M, N, K,
                                        1 if accumulate else 0), "hbsjd_gemm")
        return Cout

    def hbsjd_debug_gemm(self, A, W, Cout, accumulate=False, reps=1, acc_wait_ns=0, tile=0):
        """hbsjd_gemm `reps` times back to back; acc_wait_ns > 0 shortens the epilogue's bounded wait (time-out test)."""
        M, K = A.shape
        N = W.shape[0]
        assert W.shape[1] == K and tuple(Cout.shape) == (M, N) and Cout.dtype == self._torch.float32
        self._check(self.lib.hbsjd_debug_gemm(self.h, A.data_ptr(), W.data_ptr(), Cout.data_ptr(), M, N, K,
                                              int(accumulate), reps, acc_wait_ns, tile), "hbsjd_debug_gemm")
        return Cout

    def hbsjd_debug_fold_norm(self, on: bool):
        """RMSNorm folded into the GEMM epilogues (True) or as its own kernel (False); before the first rollout."""
        self._check(self.lib.hbsjd_debug_fold_norm(self.h, 1 if on else 0), "hbsjd_debug_fold_norm")
        self.fold_norm = bool(on)

    def hbsjd_debug_force_tile(self, tile: int):
        """Tile of every decoder GEMM of this context's forwards (0: the library's choice)."""
        self._check(self.lib.hbsjd_debug_force_tile(self.h, tile), "hbsjd_debug_force_tile")

    def hbsjd_debug_fail_round(self, rnd: int):
        """Plants a bounded wait's error in the next round with this index."""
        self._check(self.lib.hbsjd_debug_fail_round(self.h, rnd), "hbsjd_debug_fail_round")

    def hbsjd_debug_shuffle_pages(self, seed: int):
        self._check(self.lib.hbsjd_debug_shuffle_pages(self.h, seed), "hbsjd_debug_shuffle_pages")

    def hbsjd_bikl(self, logits_s, logits_t):
        """Device fp32 [rows, V] logits of two models -> device fp32 [rows] bidirectional KL (Eq. 3)."""
        out = self._torch.empty(logits_s.shape[0], dtype=self._torch.float32, device="cuda")
        assert logits_s.shape == logits_t.shape and logits_s.is_contiguous() and logits_t.is_contiguous()
        self._check(self.lib.hbsjd_bikl(self.h, logits_s.data_ptr(), logits_t.data_ptr(), logits_s.shape[0],
                                        out.data_ptr()), "hbsjd_bikl")
        return out

    def hbsjd_score(self, teacher: "Context", tokens, prefix_len, class_labels):
        """Eq. 3 on completed trajectories, this context the student.  Device int32 tensors in; returns
        (bikl_pos device fp32 [batch, T], per_image device fp32 [batch], loss float)."""
        torch = self._torch
        batch = tokens.shape[0]
        assert tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()
        assert tuple(tokens.shape) == (batch, self.shape.T)
        assert prefix_len.dtype == torch.int32 and class_labels.dtype == torch.int32
        pos = torch.empty((batch, self.shape.T), dtype=torch.float32, device="cuda")
        per = torch.empty(batch, dtype=torch.float32, device="cuda")
        loss = C.c_float(0.0)
        self._check(self.lib.hbsjd_score(self.h, teacher.h, batch, tokens.data_ptr(), prefix_len.data_ptr(),
                                         class_labels.data_ptr(), pos.data_ptr(), per.data_ptr(), C.byref(loss)),
                    "hbsjd_score")
        self.batch = 0
        teacher.batch = 0
        return pos, per, loss.value

    def hbsjd_score_topk(self, tokens, prefix_len, class_labels, k, temperature=1.0):
        """The k largest logits of this model at every position of completed trajectories: (values fp32 [batch, T, k],
        indices int32 [batch, T, k], rest fp32 [batch, T]), device tensors; empty lists for the prefixes."""
        torch = self._torch
        batch, T = tokens.shape[0], self.shape.T
        assert tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()
        assert tuple(tokens.shape) == (batch, T)
        for x in (prefix_len, class_labels):  # (read through their pointers, one per image)
            assert x.is_cuda and x.device == tokens.device and x.dtype == torch.int32 and x.is_contiguous()
            assert len(x.shape) == 1 and x.shape[0] >= batch
        values = torch.empty((batch, T, k), dtype=torch.float32, device=tokens.device)
        indices = torch.empty((batch, T, k), dtype=torch.int32, device=tokens.device)
        rest = torch.empty((batch, T), dtype=torch.float32, device=tokens.device)
        self._check(self.lib.hbsjd_score_topk(self.h, batch, tokens.data_ptr(), prefix_len.data_ptr(),
                                              class_labels.data_ptr(), k, temperature, values.data_ptr(),
                                              indices.data_ptr(), rest.data_ptr()), "hbsjd_score_topk")
        self.batch = 0
        return values, indices, rest

    def hbsjd_score_logprobs(self, tokens, prefix_len, class_labels, temperature=1.0):
        """Log-probabilities of the tokens of completed trajectories under this model, and the entropies of their distributions: (logp
        fp32 [batch, T], entropy fp32 [batch, T]), device tensors; 0 for the prefixes."""
        torch = self._torch
        batch, T = tokens.shape[0], self.shape.T
        assert tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()
        assert tuple(tokens.shape) == (batch, T)
        for x in (prefix_len, class_labels):  # (read through their pointers, one per image)
            assert x.is_cuda and x.device == tokens.device and x.dtype == torch.int32 and x.is_contiguous()
            assert len(x.shape) == 1 and x.shape[0] >= batch
        logp = torch.empty((batch, T), dtype=torch.float32, device=tokens.device)
        entropy = torch.empty_like(logp)
        self._check(self.lib.hbsjd_score_logprobs(self.h, batch, tokens.data_ptr(), prefix_len.data_ptr(), class_labels.data_ptr(),
                                                  temperature, logp.data_ptr(), entropy.data_ptr()), "hbsjd_score_logprobs")
        self.batch = 0
        return logp, entropy

    def hbsjd_destroy(self):
        if self.h:
            self.lib.hbsjd_destroy(self.h)
            self.h = C.c_void_p()

    def __del__(self):
        try:
            self.hbsjd_destroy()
        except Exception:
            pass
