"""Token operators of libsconv (include/sconv_tokens.h): layer norm from a feature map or from tokens, rotary positions
over several axes, differential attention, and their gradients.

Argument marshalling only, as in the package itself: every sum runs in the HIP kernels behind the C ABI.  Calls go to
torch's current stream; scratch that a call is not given is taken from torch's allocator for the call.  Like the package's other
calls, these are not part of torch's autograd: results do not require a gradient whatever the operands do, and a training program makes
the backward calls itself (examples/attention_block.py, or inside a torch.autograd.Function).
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import torch

from . import SconvError, _check_dev, _raw_stream, lib as _base_lib

SCONV_F32, SCONV_BF16 = 0, 1
SCONV_LAYOUT_TOKENS, SCONV_LAYOUT_MAP = 0, 1
SCONV_ROTARY_MAX_AXES, SCONV_ROTARY_MAX_PAIRS = 8, 256

_CONTIGUOUS = torch.contiguous_format
_TYPES = {torch.float32: SCONV_F32, torch.bfloat16: SCONV_BF16}
_LAYOUTS = {"tokens": SCONV_LAYOUT_TOKENS, "map": SCONV_LAYOUT_MAP}
_i32, _i64, _vp, _sz, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float


class LayerNormDesc(ctypes.Structure):
    """sconv_layernorm_desc_t"""
    _fields_ = ([(n, _i32) for n in ("N", "S", "C", "layout", "x_type", "y_type", "w_type")] + [("eps", _f32)] +
                [(n, _i64) for n in ("x_n", "x_s", "y_n", "y_s")])


class RotaryDesc(ctypes.Structure):
    """sconv_rotary_desc_t"""
    _fields_ = ([(n, _i32) for n in ("B", "S", "Hq", "Hk", "D", "type", "pairs", "axes", "interleaved", "inverse")] +
                [(n, _i64) for n in ("q_b", "q_s", "q_h", "k_b", "k_s", "k_h", "qo_b", "qo_s", "qo_h", "ko_b", "ko_s",
                                     "ko_h", "pos_b")] +
                [("axis", ctypes.c_char * SCONV_ROTARY_MAX_PAIRS)])


class DiffAttnDesc(ctypes.Structure):
    """sconv_diffattn_desc_t"""
    _fields_ = ([(n, _i32) for n in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv", "type", "causal")] + [("scale", _f32)] +
                [(n, _i64) for n in ("q_b", "q_s", "q_h", "k_b", "k_s", "k_h", "v_b", "v_s", "v_h", "mask_b")])


# Descriptors of calls seen before, by what they are made of: the tensors' shapes, strides and types and the call's numbers and switches,
# by value (nothing of the tensors themselves).  Filling one in takes longer than a small call's kernel.
_plans = {}
_PLANS_KEPT = 4096


def _number(x):
    """A number as the C call takes it.  A tensor of one element is read here, at every call: as part of a key it would stand for itself,
    whatever it came to hold."""
    return x if type(x) is float else _f32(x).value


def _sig(t):
    """What a descriptor says of a tensor."""
    if t is None:
        return None
    try:
        return t.shape, t.stride(), t.dtype, t.is_cuda
    except (AttributeError, TypeError):
        raise TypeError("tensors in device memory are wanted") from None


def _keep(key, plan):
    if len(_plans) >= _PLANS_KEPT:
        _plans.clear()
    _plans[key] = plan
    return plan


_lib = None


def _tokens_lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L, P = _base_lib(), ctypes.POINTER
        ln, ro, at = P(LayerNormDesc), P(RotaryDesc), P(DiffAttnDesc)
        L.sconv_layernorm_workspace_size.argtypes = [ln, P(_sz)]
        L.sconv_layernorm_forward.argtypes = [ln] + [_vp] * 7
        L.sconv_layernorm_backward.argtypes = [ln] + [_vp] * 9 + [_sz, _vp]
        L.sconv_rotary.argtypes = [ro] + [_vp] * 7
        L.sconv_diffattn_workspace_size.argtypes = [at, ctypes.c_int, P(_sz)]
        L.sconv_diffattn_forward.argtypes = [at] + [_vp] * 10 + [_sz, _vp]
        L.sconv_diffattn_backward.argtypes = [at] + [_vp] * 15 + [_sz, _vp]
        for f in ("sconv_layernorm_workspace_size", "sconv_layernorm_forward", "sconv_layernorm_backward", "sconv_rotary",
                  "sconv_diffattn_workspace_size", "sconv_diffattn_forward", "sconv_diffattn_backward"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(t, what, dims=None):
    """A device tensor of one of the operators' types whose last axis is contiguous; returns the type's code."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in _TYPES):
        raise TypeError(f"{what} must be an fp32 or bf16 tensor in device memory")
    if dims is not None and t.dim() != dims:
        raise ValueError(f"{what} must have {dims} axes")
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise TypeError(f"the last axis of {what} must be contiguous")
    return _TYPES[t.dtype]


def _out(t, shape, dtype, device, what):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _check_dev(t, dtype, what)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has the wrong shape")
    return t


def _opt(t):
    return None if t is None else t.data_ptr()


def _ws(ws, need, device):
    """(tensor to keep, pointer, bytes) of the scratch of a call."""
    if ws is None:
        if not need:
            return None, None, 0
        ws = torch.empty(need, dtype=torch.uint8, device=device)
    elif not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.is_contiguous()):
        raise TypeError("ws must be a contiguous tensor in device memory")
    return ws, (ws.data_ptr() if ws.numel() else None), ws.numel() * ws.element_size()


# ---- layer norm

def _rows(x, what):
    """(N, S, stride of N, stride of S) of the rows of a tokens tensor."""
    d = x.dim()
    if d == 3:
        return x.shape[0], x.shape[1], x.stride(0), x.stride(1)
    if d == 2:
        return 1, x.shape[0], 0, x.stride(0)
    if d == 1:
        return 1, 1, 0, 0
    if d == 0:
        raise ValueError(f"{what} has no axes")
    try:
        flat = x.view(-1, x.shape[-1])
    except RuntimeError:
        raise TypeError(f"the rows of {what} must lie at one stride") from None
    return 1, flat.shape[0], 0, flat.stride(0)


def _map_rows(x, what):
    """(N, places, C, stride of N, stride of C) of a feature map [N, C, H, W] or [N, C, S]."""
    if x.dim() not in (3, 4):
        raise ValueError(f"{what} must be [N, C, H, W] or [N, C, S]")
    if x.dim() == 4 and x.shape[2] > 1 and x.stride(2) != x.shape[3]:
        raise TypeError(f"the places of {what} must be contiguous")
    places = x.shape[2] if x.dim() == 3 else x.shape[2] * x.shape[3]
    return x.shape[0], places, x.shape[1], x.stride(0), x.stride(1)


def _weight_type(C, weight, bias):
    kind = None
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is None:
            continue
        code = _check(t, what, 1)
        if t.shape[0] != C:
            raise ValueError(f"{what} must be [C]")
        if kind is not None and code != kind:
            raise TypeError("weight and bias must have one type")
        kind = code
    return SCONV_F32 if kind is None else kind


def sconv_layernorm_forward(x, weight=None, bias=None, eps: float = 1e-5, layout: str = "tokens", out_dtype=None,
                            stats: bool = False, out=None):
    """Layer norm over the channels of every place: y = (x - mean) * rstd * weight + bias.

    layout "tokens": x is [..., C] and y has its shape; "map": x is a feature map [N, C, H, W] (or [N, C, S]) as
    sconv_forward leaves it and y is tokens [N, H*W, C].  out_dtype: x's type (default), or bf16 under an fp32 x.
    stats: returns (y, mean, rstd), the fp32 statistics of every place that sconv_layernorm_backward reads."""
    eps = _number(eps)
    key = (0, _sig(x), _sig(weight), _sig(bias), eps, layout, out_dtype)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _layernorm_plan(x, weight, bias, eps, layout, out_dtype))
    _, ref, shape, lead, dtype = plan
    if out is None and dtype is x.dtype and layout == "tokens":
        y = torch.empty_like(x, memory_format=_CONTIGUOUS)
    else:
        y = _out(out, shape, dtype, x.device, "out")
    mean = rstd = mp = rp = None
    if stats:
        mean = torch.empty(lead, dtype=torch.float32, device=x.device)
        rstd = torch.empty(lead, dtype=torch.float32, device=x.device)
        mp, rp = mean.data_ptr(), rstd.data_ptr()
    rc = _tokens_lib().sconv_layernorm_forward(ref, x.data_ptr(), None if weight is None else weight.data_ptr(),
                                               None if bias is None else bias.data_ptr(), y.data_ptr(), mp, rp,
                                               _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_layernorm_forward")
    return (y, mean, rstd) if stats else y


def _layernorm_plan(x, weight, bias, eps, layout, out_dtype):
    """(descriptor, reference to it, y's shape, the statistics', y's type)"""
    xt = _check(x, "x")
    if layout not in _LAYOUTS:
        raise ValueError('layout must be "tokens" or "map"')
    yt = xt if out_dtype is None else _TYPES.get(out_dtype, -1)
    if layout == "map":
        N, S, C, xn, xs = _map_rows(x, "x")
        shape, lead = (N, S, C), (N, S)
    else:
        N, S, xn, xs = _rows(x, "x")
        C, shape, lead = x.shape[-1], tuple(x.shape), tuple(x.shape[:-1])
    wt = _weight_type(C, weight, bias)
    if yt < 0:
        raise SconvError(-1, "sconv_layernorm_forward")
    desc = LayerNormDesc(N, S, C, _LAYOUTS[layout], xt, yt, wt, eps, xn, xs, S * C, C)
    return desc, ctypes.byref(desc), shape, lead, x.dtype if out_dtype is None else out_dtype


def sconv_layernorm_backward(dy, x, mean, rstd, weight=None, layout: str = "tokens", param_grads: bool = True, ws=None):
    """Gradient of sconv_layernorm_forward: (dx, dweight, dbias); dx has x's shape, layout and type, dweight and dbias
    weight's type (fp32 without one; None with param_grads False).  ws: a device tensor as scratch (optional)."""
    key = (1, _sig(dy), _sig(x), _sig(mean), _sig(rstd), _sig(weight), layout)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _layernorm_grad_plan(dy, x, mean, rstd, weight, layout))
    _, ref, C, wdtype, need = plan
    dx = torch.empty_like(x, memory_format=_CONTIGUOUS)
    dw = db = ptr = None
    nbytes = 0
    if param_grads:
        dw = torch.empty(C, dtype=wdtype, device=x.device)
        db = torch.empty(C, dtype=wdtype, device=x.device)
        ws, ptr, nbytes = _ws(ws, need, x.device)
    rc = _tokens_lib().sconv_layernorm_backward(ref, dy.data_ptr(), x.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                                None if weight is None else weight.data_ptr(), dx.data_ptr(), _opt(dw),
                                                _opt(db), ptr, nbytes, _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_layernorm_backward")
    return dx, dw, db


def _layernorm_grad_plan(dy, x, mean, rstd, weight, layout):
    """(descriptor, reference to it, channels, type of the weight's gradient, bytes of scratch)"""
    xt, yt = _check(x, "x"), _check(dy, "dy")
    if layout not in _LAYOUTS:
        raise ValueError('layout must be "tokens" or "map"')
    if layout == "map":
        N, S, C, xn, xs = _map_rows(x, "x")
        if tuple(dy.shape) != (N, S, C):
            raise ValueError("dy must be [N, places, C]")
        yn, ys = dy.stride(0), dy.stride(1)
    else:
        C = x.shape[-1] if x.dim() else 0
        if dy.shape != x.shape:
            raise ValueError("dy must have x's shape")
        N, S, xn, xs = _rows(x, "x")
        _, _, yn, ys = _rows(dy, "dy")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        _check_dev(t, torch.float32, what)
        if t.numel() != N * S:
            raise ValueError(f"{what} must have one value a place")
    desc = LayerNormDesc(N, S, C, _LAYOUTS[layout], xt, yt, _weight_type(C, weight, None), 0.0, xn, xs, yn, ys)
    need = _sz()
    rc = _tokens_lib().sconv_layernorm_workspace_size(ctypes.byref(desc), ctypes.byref(need))
    if rc:
        raise SconvError(rc, "sconv_layernorm_backward")
    return desc, ctypes.byref(desc), C, torch.float32 if weight is None else weight.dtype, need.value


# ---- rotary positions

def sconv_rotary_axes(sections: Sequence[int]) -> bytes:
    """The axis of every pair where axis a turns sections[a] pairs in a row: sconv_rotary_axes((16, 16)) for the rows and
    columns of a map under heads of 64."""
    if not sections or min(sections) < 0:
        raise ValueError("sections must be counts of pairs")
    return bytes(a for a, n in enumerate(sections) for _ in range(n))


def _rotary(q, k, positions, freq, axes, interleaved, inverse, out, what):
    if type(axes) is not bytes:
        axes = bytes(list(axes))
    interleaved = bool(interleaved)
    key = (2 + inverse, _sig(q), _sig(k), _sig(positions), _sig(freq), axes, interleaved)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _rotary_plan(q, k, positions, freq, axes, interleaved, inverse, what))
    _, ref = plan
    ko = kp = kop = None
    if out is None:
        qo = torch.empty_like(q, memory_format=_CONTIGUOUS)
        if k is not None:
            ko = torch.empty_like(k, memory_format=_CONTIGUOUS)
    else:
        qo = _out(out[0], q.shape, q.dtype, q.device, "out[0]")
        if k is not None:
            ko = _out(out[1], k.shape, k.dtype, k.device, "out[1]")
    if k is not None:
        kp, kop = k.data_ptr(), ko.data_ptr()
    rc = _tokens_lib().sconv_rotary(ref, q.data_ptr(), kp, positions.data_ptr(), freq.data_ptr(), qo.data_ptr(), kop,
                                    _raw_stream(torch))
    if rc:
        raise SconvError(rc, what)
    return qo, ko


def _rotary_plan(q, k, positions, freq, axes, interleaved, inverse, what):
    """(descriptor, reference to it)"""
    qt = _check(q, "q", 4)
    B, S, Hq, D = q.shape
    Hk = 0
    if k is not None:
        if _check(k, "k", 4) != qt:
            raise TypeError("q and k must have one type")
        if k.shape[0] != B or k.shape[1] != S or k.shape[3] != D:
            raise ValueError("k must be [B, S, heads, D] as q is")
        Hk = k.shape[2]
    _check_dev(freq, torch.float32, "inv_freq")
    _check_dev(positions, torch.int32, "positions")
    pairs = len(axes)
    batch = positions.shape[0] if positions.dim() == 3 else 1
    if positions.dim() not in (2, 3) or batch not in (1, B) or positions.shape[-2] != S:
        raise ValueError("positions must be [B or 1, S, axes] or [S, axes]")
    n_axes = positions.shape[-1]
    if freq.dim() != 1 or freq.shape[0] != pairs:
        raise ValueError("inv_freq must have one value a pair, as axes has")
    if pairs > SCONV_ROTARY_MAX_PAIRS:
        raise SconvError(-2, what)
    desc = RotaryDesc(B, S, Hq, Hk, D, qt, pairs, n_axes, 1 if interleaved else 0, inverse, q.stride(0), q.stride(1),
                      q.stride(2), 0, 0, 0, S * Hq * D, Hq * D, D, S * Hk * D, Hk * D, D, S * n_axes if batch > 1 else 0)
    if Hk:
        desc.k_b, desc.k_s, desc.k_h = k.stride(0), k.stride(1), k.stride(2)
    ctypes.memmove(ctypes.addressof(desc) + RotaryDesc.axis.offset, axes, pairs)
    return desc, ctypes.byref(desc)


def sconv_rotary_forward(q, k, positions, inv_freq, axes: bytes, interleaved: bool = False, out=None):
    """Rotary positions over several axes: pair p of every head turns by positions[..., axes[p]] * inv_freq[p].

    q [B, S, Hq, D] and k [B, S, Hk, D] (or None) share one launch; both may be slices of a projection's output.
    positions: int32 [B or 1, S, number of axes]; inv_freq: fp32, one value a pair; axes: the axis of every pair
    (sconv_rotary_axes).  Pair p is elements p and p + pairs, interleaved 2p and 2p + 1; elements beyond the pairs are
    copied.  out: (for q, for k), contiguous, may be q and k themselves.  Returns (q turned, k turned or None)."""
    return _rotary(q, k, positions, inv_freq, axes, interleaved, 0, out, "sconv_rotary_forward")


def sconv_rotary_backward(dq, dk, positions, inv_freq, axes: bytes, interleaved: bool = False, out=None):
    """Gradient of sconv_rotary_forward: the turn by the opposite angles."""
    return _rotary(dq, dk, positions, inv_freq, axes, interleaved, 1, out, "sconv_rotary_backward")


# ---- differential attention

def _attn_plan(q, k, v, lam, scale, causal, k_lengths, k_mask):
    """(descriptor, reference to it, out's shape, lse's, bytes of scratch forward and backward)"""
    if scale is not None:
        scale = _number(scale)
    causal = bool(causal)
    key = (4, _sig(q), _sig(k), _sig(v), _sig(lam), scale, causal, _sig(k_lengths), _sig(k_mask))
    plan = _plans.get(key)
    if plan is None:
        desc = _attn_desc(q, k, v, lam, scale, causal, k_lengths, k_mask)
        need = [_sz(), _sz()]
        for backward in (0, 1):
            rc = _tokens_lib().sconv_diffattn_workspace_size(ctypes.byref(desc), backward, ctypes.byref(need[backward]))
            if rc:
                raise SconvError(rc, "sconv_diffattn")
        plan = _keep(key, (desc, ctypes.byref(desc), (desc.B, desc.Sq, desc.H, desc.Dv), (2, desc.B, desc.H, desc.Sq),
                           need[0].value, need[1].value))
    return plan


def _attn_desc(q, k, v, lam, scale, causal, k_lengths, k_mask):
    qt = _check(q, "q", 4)
    if _check(k, "k", 4) != qt or _check(v, "v", 4) != qt:
        raise TypeError("q, k and v must have one type")
    B, Sq, H2, D = q.shape
    _, Sk, Hkv2, _ = k.shape
    H, Hkv = H2 // 2, Hkv2 // 2
    if H2 % 2 or Hkv2 % 2 or k.shape[0] != B or k.shape[3] != D or v.shape[0] != B or v.shape[1] != Sk or v.shape[2] != Hkv:
        raise ValueError("q must be [B, Sq, 2H, D], k [B, Sk, 2Hkv, D], v [B, Sk, Hkv, Dv]")
    _check_dev(lam, torch.float32, "lam")
    if lam.dim() != 1 or lam.shape[0] != H:
        raise ValueError("lam must be [H]")
    mask_b = 0
    if k_lengths is not None:
        _check_dev(k_lengths, torch.int32, "k_lengths")
        if k_lengths.dim() != 1 or k_lengths.shape[0] != B:
            raise ValueError("k_lengths must be [B]")
    if k_mask is not None:
        if not (isinstance(k_mask, torch.Tensor) and k_mask.is_cuda and k_mask.dtype in (torch.bool, torch.uint8)):
            raise TypeError("k_mask must be a bool or uint8 tensor in device memory")
        if k_mask.dim() != 2 or k_mask.shape[0] != B or k_mask.shape[1] != Sk:
            raise ValueError("k_mask must be [B, Sk]")
        if Sk > 1 and k_mask.stride(1) != 1:
            raise TypeError("the last axis of k_mask must be contiguous")
        mask_b = k_mask.stride(0)
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    return DiffAttnDesc(B, Sq, Sk, H, Hkv, D, v.shape[3], qt, 1 if causal else 0,
                        (1.0 / math.sqrt(D) if D else 0.0) if scale is None else scale, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
                        vs[0], vs[1], vs[2], mask_b)


def sconv_diffattn_workspace_size(q, k, v, lam, backward: bool = False) -> int:
    """Bytes of scratch that a call on these tensors can use (forward) or needs (backward)."""
    return _attn_plan(q, k, v, lam, None, False, None, None)[5 if backward else 4]


def sconv_diffattn_forward(q, k, v, lam, scale: Optional[float] = None, causal: bool = False, k_lengths=None, k_mask=None,
                           save: bool = False, out=None, ws=None):
    """Differential attention: out = (softmax(scale Q1 K1^T) - lam softmax(scale Q2 K2^T)) V for every head.

    q [B, Sq, 2H, D] (queries of the two maps at heads 2h, 2h + 1), k [B, Sk, 2Hkv, D], v [B, Sk, Hkv, Dv], H a multiple
    of Hkv; lam: fp32 [H]; scale: a number, 1/sqrt(D) by default (a tensor of one element is read by the host).  k_lengths: int32 [B], keys of every request; k_mask: bool or
    uint8 [B, Sk], false where a key is not to be seen; causal: the last query stands at the request's last key.  A query
    that sees nothing gives zeros.  One token over a cache is the same call with Sq = 1 and k, v the cache.  Returns out
    [B, Sq, H, Dv]; save: (out, second, lse), the last two for sconv_diffattn_backward.  ws: a device tensor as
    scratch for calls of few queries (by default torch's allocator is asked)."""
    _, ref, shape, lse_shape, need, _ = _attn_plan(q, k, v, lam, scale, causal, k_lengths, k_mask)
    out = _out(out, shape, q.dtype, q.device, "out")
    second = lse = sp = lp = None
    if save:
        second = torch.empty(shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(lse_shape, dtype=torch.float32, device=q.device)
        sp, lp = second.data_ptr(), lse.data_ptr()
    ws, ptr, nbytes = _ws(ws, need, q.device)
    rc = _tokens_lib().sconv_diffattn_forward(ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), lam.data_ptr(), _opt(k_lengths),
                                              _opt(k_mask), out.data_ptr(), sp, lp, ptr, nbytes, _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_diffattn_forward")
    return (out, second, lse) if save else out


def sconv_diffattn_backward(dout, q, k, v, lam, out, second, lse, scale: Optional[float] = None, causal: bool = False,
                            k_lengths=None, k_mask=None, ws=None):
    """Gradient of sconv_diffattn_forward: (dq, dk, dv, dlam), contiguous, in the shapes and types of q, k, v, lam.
    out, second, lse: what the forward call returned with save; the other arguments as they were given to it."""
    _, ref, shape, lse_shape, _, need = _attn_plan(q, k, v, lam, scale, causal, k_lengths, k_mask)
    for t, what in ((dout, "dout"), (out, "out"), (second, "second")):
        _check_dev(t, q.dtype, what)
        if t.shape != shape:
            raise ValueError(f"{what} must be [B, Sq, H, Dv]")
    _check_dev(lse, torch.float32, "lse")
    if lse.shape != lse_shape:
        raise ValueError("lse must be [2, B, H, Sq]")
    dq, dk, dv, dlam = (torch.empty_like(t, memory_format=_CONTIGUOUS) for t in (q, k, v, lam))
    ws, ptr, nbytes = _ws(ws, need, q.device)
    rc = _tokens_lib().sconv_diffattn_backward(ref, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), lam.data_ptr(),
                                               _opt(k_lengths), _opt(k_mask), out.data_ptr(), second.data_ptr(),
                                               lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dlam.data_ptr(),
                                               ptr, nbytes, _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_diffattn_backward")
    return dq, dk, dv, dlam
