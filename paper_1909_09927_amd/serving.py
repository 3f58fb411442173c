"""Serving operators of libsconv (include/sconv_serving.h): a step of an attention block in 8 bits - root-mean-square norm with the
residual's addition (and its gradient), 8-bit operands with block scales, their product, a paged cache of keys and values, and
differential attention of new tokens over it.

Argument marshalling only, as in tokens.py, whose conventions hold here: calls go to torch's current stream of the current
device, which has to be the tensors', scratch that a call is not given is taken from torch's allocator for the call, and the calls
are not part of torch's autograd.

8-bit values travel as a pair (values, scales): torch.float8_e4m3fn and uint8; scale byte s stands for 2^(s - 127).
"""
from __future__ import annotations

import ctypes
import math
from operator import index
from typing import NamedTuple, Optional

import torch

from . import SconvError, _raw_stream, lib as _base_lib
from .tokens import SCONV_BF16, SCONV_F32, _TYPES, _keep, _number, _plans, _ws

SCONV_E4M3, SCONV_SCALE_BLOCK = 2, 128
E4M3 = torch.float8_e4m3fn

_KINDS = {**_TYPES, E4M3: SCONV_E4M3}
_i32, _i64, _vp, _sz, _f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float


class RmsNormDesc(ctypes.Structure):
    """sconv_rmsnorm_desc_t"""
    _fields_ = ([(n, _i32) for n in ("rows", "C", "x_type", "t_type", "y_type", "w_type")] + [("eps", _f32)] +
                [(n, _i64) for n in ("x_r", "res_r", "t_r", "y_r")])


class Quant8Desc(ctypes.Structure):
    """sconv_quant8_desc_t"""
    _fields_ = [(n, _i32) for n in ("M", "K", "type", "block_rows")] + [(n, _i64) for n in ("x_m", "q_m")]


class Linear8Desc(ctypes.Structure):
    """sconv_linear8_desc_t"""
    _fields_ = [(n, _i32) for n in ("M", "N", "K", "y_type")] + [(n, _i64) for n in ("x_m", "w_n", "y_m")] + [("exact", _i32)]


class PagesDesc(ctypes.Structure):
    """sconv_pages_t"""
    _fields_ = ([(n, _i32) for n in ("pages", "page_size", "table_width", "type", "Hk", "D", "Hv", "Dv")] +
                [(n, _i64) for n in ("k_p", "k_s", "k_h", "v_p", "v_s", "v_h", "ks_p", "ks_s", "ks_h", "vs_p", "vs_s", "vs_h",
                                     "table_b")])


class PagesDev(ctypes.Structure):
    """sconv_pages_dev_t"""
    _fields_ = [(n, _vp) for n in ("k", "v", "ks", "vs", "table")]


class CacheDesc(ctypes.Structure):
    """sconv_cache_desc_t"""
    _fields_ = ([(n, _i32) for n in ("B", "S", "type")] + [(n, _i64) for n in ("k_b", "k_s", "k_h", "v_b", "v_s", "v_h")] +
                [("pages", PagesDesc)])


class PagedDesc(ctypes.Structure):
    """sconv_paged_desc_t"""
    _fields_ = ([(n, _i32) for n in ("B", "Sq", "H", "Hkv", "type", "causal")] + [("scale", _f32)] +
                [(n, _i64) for n in ("q_b", "q_s", "q_h")] + [("pages", PagesDesc)])


class PagedCache(NamedTuple):
    """A paged cache: k [pages, page_size, key heads, D], v [pages, page_size, value heads, Dv] (of the tokens' type, or
    float8_e4m3fn with k_scales [pages, page_size, key heads] and v_scales), table int32 [requests, width]: position p of request b
    stands in slot p % page_size of page table[b, p // page_size]; an entry outside 0 .. pages - 1 is a page that is not there.
    All may be strided but for the last axis of k, v and table."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    k_scales: Optional[torch.Tensor] = None
    v_scales: Optional[torch.Tensor] = None


_lib = None


def _serving_lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L, P = _base_lib(), ctypes.POINTER
        rn, ca, at, dev = P(RmsNormDesc), P(CacheDesc), P(PagedDesc), P(PagesDev)
        L.sconv_rmsnorm_workspace_size.argtypes = [rn, P(_sz)]
        L.sconv_rmsnorm_forward.argtypes = [rn] + [_vp] * 8
        L.sconv_rmsnorm_backward.argtypes = [rn] + [_vp] * 9 + [_sz, _vp]
        L.sconv_quant8.argtypes = [P(Quant8Desc)] + [_vp] * 4
        L.sconv_linear8.argtypes = [P(Linear8Desc)] + [_vp] * 6
        L.sconv_cache_write.argtypes = [ca] + [_vp] * 4 + [dev, _vp]
        L.sconv_cache_read.argtypes = [ca, dev] + [_vp] * 5
        L.sconv_diffattn_paged.argtypes = [at, _vp, dev] + [_vp] * 4 + [_sz, _vp]
        L.sconv_diffattn_paged_workspace_size.argtypes = [at, P(_sz)]
        for f in ("sconv_rmsnorm_workspace_size", "sconv_rmsnorm_forward", "sconv_rmsnorm_backward", "sconv_quant8", "sconv_linear8",
                  "sconv_cache_write", "sconv_cache_read", "sconv_diffattn_paged", "sconv_diffattn_paged_workspace_size"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def _sig(t):
    """What a descriptor says of a tensor, and where it is."""
    if t is None:
        return None
    try:
        return t.shape, t.stride(), t.dtype, t.device
    except (AttributeError, TypeError):
        raise TypeError("tensors in device memory are wanted") from None


def _current(device):
    """Calls go to the current device's stream."""
    if device.index != torch._C._cuda_getDevice():
        raise ValueError(f"the tensors are on {device}, which is not the current device")


def _check(t, what, kinds, dims=None, device=None):
    """A device tensor of one of the types whose last axis is contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in kinds):
        raise TypeError(f"{what} must be a tensor of {' or '.join(str(k)[6:] for k in kinds)} in device memory")
    if dims is not None and t.dim() != dims:
        raise ValueError(f"{what} must have {dims} axes")
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise TypeError(f"the last axis of {what} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on another device")
    return _KINDS.get(t.dtype)


def _vector(t, what, dtype, n, device):
    _check(t, what, (dtype,), 1, device)
    if t.shape[0] != n:
        raise ValueError(f"{what} must be [{n}]")


def _rows(x, what):
    """(rows, their stride) of a tensor [..., C]."""
    d = x.dim()
    if d == 2:
        return x.shape[0], x.stride(0)
    if d == 1:
        return 1, 0
    if d == 0:
        raise ValueError(f"{what} has no axes")
    if x.numel() == 0:
        return math.prod(x.shape[:-1]), x.shape[-1]
    try:
        flat = x.view(-1, x.shape[-1])
    except RuntimeError:
        raise TypeError(f"the rows of {what} must lie at one stride") from None
    return flat.shape[0], flat.stride(0)


def _blocks(n):
    return (n + SCONV_SCALE_BLOCK - 1) // SCONV_SCALE_BLOCK


def _opt(t):
    return None if t is None else t.data_ptr()


def _given(t, shape, dtype, device, what):
    """A contiguous result that the caller brought."""
    if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype and t.is_contiguous()):
        raise TypeError(f"{what} must be a contiguous {dtype} tensor on the operands' device")
    if t.shape != torch.Size(shape):
        raise ValueError(f"{what} has the wrong shape")
    return t


# ---- root-mean-square norm

def sconv_rmsnorm_forward(x, weight=None, residual=None, eps: float = 1e-6, out_dtype=None, stats: bool = False, total=None, out=None):
    """Root-mean-square norm of rows [..., C] with a residual stream's addition: t = x + residual, y = t / rms(t) * weight.

    residual: of x's shape, its type or fp32 over a bf16 x.  out_dtype: x's type (default), bf16, or float8_e4m3fn for what
    sconv_linear8 reads: y is then (values, scales [..., ceil(C / 128)]).  Returns (y, t, rstd): t, of residual's type, without a
    residual None; rstd, fp32, with stats (sconv_rmsnorm_backward reads it), otherwise None.  total: where t is to go, may be residual itself;
    out: where y is to go (8 bits: a pair)."""
    eps = _number(eps)
    key = (10, _sig(x), _sig(weight), _sig(residual), _sig(total), eps, out_dtype)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _rmsnorm_plan(x, weight, residual, total, eps, out_dtype))
    _, ref, dtype, shape, blocks, device = plan
    _current(device)
    scales = sp = None
    if dtype is E4M3:
        if out is None:
            y, scales = x.new_empty(shape, dtype=E4M3), x.new_empty(blocks, dtype=torch.uint8)
        else:
            y, scales = _given(out[0], shape, E4M3, device, "out[0]"), _given(out[1], blocks, torch.uint8, device, "out[1]")
        sp = scales.data_ptr()
    elif out is None:
        y = x.new_empty(shape, dtype=dtype)
    else:
        y = _given(out, shape, dtype, device, "out")
    if residual is not None and total is None:
        total = residual.new_empty(shape)
    rstd = x.new_empty(shape[:-1], dtype=torch.float32) if stats else None
    rc = _serving_lib().sconv_rmsnorm_forward(ref, x.data_ptr(), _opt(residual), _opt(weight), y.data_ptr(), sp, _opt(total), _opt(rstd),
                                              _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_rmsnorm_forward")
    return (y if scales is None else (y, scales)), total, rstd


def _rmsnorm_plan(x, weight, residual, total, eps, out_dtype):
    """(descriptor, reference to it, y's type, its shape and its scales', device)"""
    xt = _check(x, "x", _TYPES)
    rows, xr = _rows(x, "x")
    C = x.shape[-1]
    tt, res_r, t_r = xt, 0, C
    if residual is not None:
        tt = _check(residual, "residual", _TYPES, None, x.device)
        if residual.shape != x.shape:
            raise ValueError("residual must have x's shape")
        _, res_r = _rows(residual, "residual")
    if total is not None:
        if residual is None:
            raise ValueError("total is for calls with a residual")
        if _check(total, "total", _TYPES, None, x.device) != tt or total.shape != x.shape:
            raise TypeError("total must have residual's shape and type")
        _, t_r = _rows(total, "total")
        if rows > 1 and t_r < C:
            raise ValueError("the rows of total must lie apart")
    wt = SCONV_F32
    if weight is not None:
        wt = _check(weight, "weight", _TYPES, 1, x.device)
        if weight.shape[0] != C:
            raise ValueError("weight must be [C]")
    dtype = x.dtype if out_dtype is None else out_dtype
    yt = _KINDS.get(dtype, -1)
    desc = RmsNormDesc(rows, C, xt, tt, yt, wt, eps, xr, res_r, t_r, C)
    return desc, ctypes.byref(desc), dtype, tuple(x.shape), (*x.shape[:-1], _blocks(C)), x.device


def sconv_rmsnorm_backward(dy, total, rstd, weight=None, dtotal=None, x_dtype=None, param_grads: bool = True, ws=None):
    """Gradient of sconv_rmsnorm_forward: (dx, dresidual, dweight).

    dy: of total's shape, in y's type as the forward call gives it: bf16, or fp32 where x is fp32; total: the sum that the forward call
    returned (without a residual: x); dtotal: the gradient that reaches the sum along the stream, in total's type (optional).  x and residual have
    one gradient, in total's type; x_dtype: x's type where it is bf16 under an fp32 stream (dx is then its rounding, dy is bf16).  dweight: weight's type (fp32 without one; None
    with param_grads False).  ws: a device tensor as scratch (optional)."""
    key = (11, _sig(dy), _sig(total), _sig(rstd), _sig(weight), _sig(dtotal), x_dtype)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _rmsnorm_grad_plan(dy, total, rstd, weight, dtotal, x_dtype))
    _, ref, shape, need, device = plan
    _current(device)
    dres = total.new_empty(shape)
    narrow = x_dtype is not None and x_dtype != total.dtype
    dx = total.new_empty(shape, dtype=x_dtype) if narrow else None
    dw = ptr = None
    nbytes = 0
    if param_grads:
        dw = total.new_empty(shape[-1:], dtype=torch.float32 if weight is None else weight.dtype)
        ws, ptr, nbytes = _ws(ws, need, device)
    rc = _serving_lib().sconv_rmsnorm_backward(ref, dy.data_ptr(), total.data_ptr(), rstd.data_ptr(), _opt(weight), _opt(dtotal), _opt(dx),
                                               dres.data_ptr(), _opt(dw), ptr, nbytes, _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_rmsnorm_backward")
    return (dx if narrow else dres), dres, dw


def _rmsnorm_grad_plan(dy, total, rstd, weight, dtotal, x_dtype):
    """(descriptor, reference to it, the gradients' shape, bytes of scratch, device)"""
    tt = _check(total, "total", _TYPES)
    yt = _check(dy, "dy", _TYPES, None, total.device)
    if dy.shape != total.shape:
        raise ValueError("dy must have total's shape")
    rows, t_r = _rows(total, "total")
    _, y_r = _rows(dy, "dy")
    C, res_r = total.shape[-1], 0
    xt = tt if x_dtype is None else _TYPES.get(x_dtype, -1)
    _check(rstd, "rstd", (torch.float32,), None, total.device)
    if not rstd.is_contiguous() or rstd.numel() != rows:
        raise ValueError("rstd must have one value a row")
    if dtotal is not None:
        if _check(dtotal, "dtotal", _TYPES, None, total.device) != tt or dtotal.shape != total.shape:
            raise TypeError("dtotal must have total's shape and type")
        _, res_r = _rows(dtotal, "dtotal")
    wt = SCONV_F32
    if weight is not None:
        wt = _check(weight, "weight", _TYPES, 1, total.device)
        if weight.shape[0] != C:
            raise ValueError("weight must be [C]")
    desc = RmsNormDesc(rows, C, xt, tt, yt, wt, 0.0, 0, res_r, t_r, y_r)
    need = _sz()
    rc = _serving_lib().sconv_rmsnorm_workspace_size(ctypes.byref(desc), ctypes.byref(need))
    if rc:
        raise SconvError(rc, "sconv_rmsnorm_backward")
    return desc, ctypes.byref(desc), tuple(total.shape), need.value, total.device


# ---- 8-bit operands and their product

def sconv_quant8(x, block_rows: int = 1, out=None):
    """Rows [..., K] into 8 bits: (values, scales), a scale for every 128 of a row ([..., ceil(K / 128)]), or with block_rows 128 for
    128 x 128 of weights [N, K] ([ceil(N / 128), ceil(K / 128)]).  out: a pair (optional)."""
    block_rows = index(block_rows)
    key = (12, _sig(x), block_rows)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _quant8_plan(x, block_rows))
    _, ref, shape, blocks, device = plan
    _current(device)
    if out is None:
        q, s = x.new_empty(shape, dtype=E4M3), x.new_empty(blocks, dtype=torch.uint8)
    else:
        q, s = _given(out[0], shape, E4M3, device, "out[0]"), _given(out[1], blocks, torch.uint8, device, "out[1]")
    rc = _serving_lib().sconv_quant8(ref, x.data_ptr(), q.data_ptr(), s.data_ptr(), _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_quant8")
    return q, s


def _quant8_plan(x, block_rows):
    """(descriptor, reference to it, the values' shape and the scales', device)"""
    xt = _check(x, "x", _TYPES, 2 if block_rows != 1 else None)
    M, x_m = _rows(x, "x")
    K = x.shape[-1]
    desc = Quant8Desc(M, K, xt, block_rows, x_m, K)
    blocks = (*x.shape[:-1], _blocks(K)) if block_rows == 1 else (_blocks(M), _blocks(K))
    return desc, ctypes.byref(desc), tuple(x.shape), blocks, x.device


def sconv_linear8(x, w, out_dtype=torch.bfloat16, out=None, exact: bool = False):
    """Product of 8-bit operands: y[..., n] = sum_k x[..., k] w[n, k], both as the values that they stand for.

    x: (values [..., K], scales [..., ceil(K / 128)]), as sconv_quant8(x) and sconv_rmsnorm_forward give them; w: (values [N, K], scales
    [ceil(N / 128), ceil(K / 128)]), sconv_quant8(weights, 128) once.  out_dtype: bf16 or fp32.  exact: exact products for bf16 results of more
    than 64 rows, too (fp32 ones always have them); without it the matrix pipe cuts off what is far below the largest of eight."""
    (xv, xs), (wv, wsc) = x, w
    exact = bool(exact)
    key = (13, _sig(xv), _sig(xs), _sig(wv), _sig(wsc), out_dtype, exact)
    plan = _plans.get(key)
    if plan is None:
        plan = _keep(key, _linear8_plan(xv, xs, wv, wsc, out_dtype, exact))
    _, ref, shape, device = plan
    _current(device)
    y = xv.new_empty(shape, dtype=out_dtype) if out is None else _given(out, shape, out_dtype, device, "out")
    rc = _serving_lib().sconv_linear8(ref, xv.data_ptr(), xs.data_ptr(), wv.data_ptr(), wsc.data_ptr(), y.data_ptr(), _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_linear8")
    return y


def _linear8_plan(xv, xs, wv, wsc, out_dtype, exact):
    """(descriptor, reference to it, y's shape, device)"""
    _check(xv, "x's values", (E4M3,))
    _check(wv, "w's values", (E4M3,), 2, xv.device)
    M, x_m = _rows(xv, "x")
    (N, K), w_n = wv.shape, wv.stride(0)
    if xv.shape[-1] != K:
        raise ValueError("x and w must have one depth K")
    for s, shape, what in ((xs, (*xv.shape[:-1], _blocks(K)), "x's scales"), (wsc, (_blocks(N), _blocks(K)), "w's scales")):
        _check(s, what, (torch.uint8,), None, xv.device)
        if s.shape != torch.Size(shape) or not s.is_contiguous():
            raise ValueError(f"{what} must be contiguous, of shape {shape}")
    desc = Linear8Desc(M, N, K, _TYPES.get(out_dtype, -1), x_m, w_n, N, exact)
    return desc, ctypes.byref(desc), (*xv.shape[:-1], N), xv.device


# ---- a paged cache

def sconv_cache_new(requests: int, width: int, pages: int, page_size: int, key_heads: int, head: int, value_heads: int, value_head: int,
                    dtype=E4M3, device="cuda") -> PagedCache:
    """An empty cache (its table knows no pages: -1).  A page holds head after head, so that a head's slots lie beside each other."""
    def heads_first(n, *last, dtype=dtype):
        return torch.zeros(pages, n, page_size, *last, dtype=dtype, device=device).transpose(1, 2)

    quantised = dtype == E4M3
    return PagedCache(heads_first(key_heads, head), heads_first(value_heads, value_head),
                      torch.full((requests, width), -1, dtype=torch.int32, device=device),
                      heads_first(key_heads, dtype=torch.uint8) if quantised else None,
                      heads_first(value_heads, dtype=torch.uint8) if quantised else None)


def _pages_desc(cache, kind, B):
    """PagesDesc of a cache that serves tokens of a type."""
    k, v, table, ks, vs = cache
    kt = _check(k, "the cache's k", _KINDS, 4)
    if _check(v, "the cache's v", _KINDS, 4, k.device) != kt or v.shape[:2] != k.shape[:2]:
        raise ValueError("the cache's k and v must be [pages, page_size, heads, width] of one type")
    if kt != kind and kt != SCONV_E4M3:
        raise TypeError("the cache must be of the tokens' type or float8_e4m3fn")
    _check(table, "the cache's table", (torch.int32,), 2, k.device)
    if table.shape[0] != B:
        raise ValueError("the cache's table must have a row for every request")
    strides = [0] * 6
    if kt == SCONV_E4M3:
        for i, (s, of, what) in enumerate(((ks, k, "k_scales"), (vs, v, "v_scales"))):
            if not (isinstance(s, torch.Tensor) and s.device == k.device and s.dtype == torch.uint8 and s.shape == of.shape[:3]):
                raise TypeError(f"the cache's {what} must be uint8 [pages, page_size, heads]")
            strides[3 * i:3 * i + 3] = s.stride()
    elif ks is not None or vs is not None:
        raise ValueError("scales are for caches of float8_e4m3fn")
    return PagesDesc(k.shape[0], k.shape[1], table.shape[1], kt, k.shape[2], k.shape[3], v.shape[2], v.shape[3], *k.stride()[:3],
                     *v.stride()[:3], *strides, table.stride(0))


def _pages_dev(cache):
    k, v, table, ks, vs = cache
    return ctypes.byref(PagesDev(k.data_ptr(), v.data_ptr(), _opt(ks), _opt(vs), table.data_ptr()))


def _cache_sig(cache):
    k, v, table, ks, vs = cache
    return _sig(k), _sig(v), _sig(table), _sig(ks), _sig(vs)


def _cache_plan(cache, k, v, starts, counts):
    """(descriptor, reference to it, device)"""
    key = (14, _cache_sig(cache), _sig(k), _sig(v), _sig(starts), _sig(counts))
    plan = _plans.get(key)
    if plan is None:
        kt = _check(k, "k", _TYPES, 4)
        if _check(v, "v", _TYPES, 4, k.device) != kt or v.shape[:2] != k.shape[:2]:
            raise ValueError("k and v must be [B, S, heads, width] of one type")
        B, S = k.shape[:2]
        pages = _pages_desc(cache, kt, B)
        if cache.k.device != k.device:
            raise ValueError("the cache is on another device")
        if k.shape[2:] != cache.k.shape[2:] or v.shape[2:] != cache.v.shape[2:]:
            raise ValueError("k and v must have the cache's heads and widths")
        _vector(starts, "starts", torch.int32, B, k.device)
        if counts is not None:
            _vector(counts, "counts", torch.int32, B, k.device)
        desc = CacheDesc(B, S, kt, *k.stride()[:3], *v.stride()[:3], pages)
        plan = _keep(key, (desc, ctypes.byref(desc), k.device))
    return plan


def sconv_cache_write(cache: PagedCache, k, v, starts, counts=None) -> None:
    """Writes new tokens' keys and values into their requests' pages, in 8 bits where the cache is.

    k [B, S, key heads, D], v [B, S, value heads, Dv], may be slices of a projection's output; token i < counts[b] (int32, S by default) of
    request b goes to position starts[b] + i (int32).  Positions without a page, and rows behind counts, write nothing; no two tokens of a call
    may have one slot."""
    _, ref, device = _cache_plan(cache, k, v, starts, counts)
    _current(device)
    rc = _serving_lib().sconv_cache_write(ref, k.data_ptr(), v.data_ptr(), starts.data_ptr(), _opt(counts), _pages_dev(cache), _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_cache_write")


def sconv_cache_read(cache: PagedCache, S: int, starts, counts=None, out_dtype=None, out=None):
    """Positions starts[b] + i, i < counts[b] (S by default), of every request out of its pages: (k [B, S, key heads, D], v [B, S, value
    heads, Dv]), contiguous; rows that are not there are zeros.  out_dtype: the cache's type; of an 8-bit cache bf16 (default, exact) or fp32."""
    k, v = cache.k, cache.v
    S = index(S)
    if out is None:
        key = (16, _cache_sig(cache), S, _sig(starts), _sig(counts), out_dtype)
        plan = _plans.get(key)
        if plan is None:
            dtype = out_dtype or (torch.bfloat16 if k.dtype == E4M3 else k.dtype)
            B = starts.shape[0]
            out = k.new_empty((B, S, *k.shape[2:]), dtype=dtype), v.new_empty((B, S, *v.shape[2:]), dtype=dtype)
            plan = _keep(key, (*_cache_plan(cache, *out, starts, counts), tuple(out[0].shape), tuple(out[1].shape), dtype))
        else:
            out = k.new_empty(plan[3], dtype=plan[5]), v.new_empty(plan[4], dtype=plan[5])
    else:
        plan = _cache_plan(cache, out[0], out[1], starts, counts)
    ref, device = plan[1:3]
    _current(device)
    rc = _serving_lib().sconv_cache_read(ref, _pages_dev(cache), starts.data_ptr(), _opt(counts), out[0].data_ptr(), out[1].data_ptr(),
                                         _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_cache_read")
    return out


# ---- attention over it

def _paged_plan(q, cache, lam, lengths, scale, causal):
    """(descriptor, reference to it, out's shape, bytes of scratch, device)"""
    if scale is not None:
        scale = _number(scale)
    causal = bool(causal)
    key = (15, _sig(q), _cache_sig(cache), _sig(lam), _sig(lengths), scale, causal)
    plan = _plans.get(key)
    if plan is None:
        qt = _check(q, "q", _TYPES, 4)
        B, Sq, H2, D = q.shape
        pages = _pages_desc(cache, qt, B)
        if cache.k.device != q.device:
            raise ValueError("the cache is on another device")
        Hkv = cache.v.shape[2]
        if H2 % 2 or cache.k.shape[2] != 2 * Hkv or cache.k.shape[3] != D:
            raise ValueError("q must be [B, Sq, 2H, D], the cache's k [pages, page_size, 2Hkv, D], its v [pages, page_size, Hkv, Dv]")
        _vector(lam, "lam", torch.float32, H2 // 2, q.device)
        _vector(lengths, "lengths", torch.int32, B, q.device)
        desc = PagedDesc(B, Sq, H2 // 2, Hkv, qt, 1 if causal else 0, (1.0 / math.sqrt(D) if D else 0.0) if scale is None else scale,
                         *q.stride()[:3], pages)
        need = _sz()
        rc = _serving_lib().sconv_diffattn_paged_workspace_size(ctypes.byref(desc), ctypes.byref(need))
        if rc:
            raise SconvError(rc, "sconv_diffattn_paged")
        plan = _keep(key, (desc, ctypes.byref(desc), (B, Sq, H2 // 2, cache.v.shape[3]), need.value, q.device))
    return plan


def sconv_diffattn_paged_workspace_size(q, cache: PagedCache, lam, lengths) -> int:
    """Bytes of scratch that a call on these tensors can use."""
    return _paged_plan(q, cache, lam, lengths, None, False)[3]


def sconv_diffattn_paged(q, cache: PagedCache, lam, lengths, scale: Optional[float] = None, causal: bool = False, out=None, ws=None):
    """Differential attention (sconv_diffattn_forward) of new tokens over a paged cache: [B, Sq, H, Dv].

    q [B, Sq, 2H, D]; the cache's k [pages, page_size, 2Hkv, D], its v [pages, page_size, Hkv, Dv], H a multiple of Hkv; lam: fp32 [H];
    lengths: int32 [B], positions of every request, the new tokens' among them; causal: the last query stands at the last position.  A query
    that sees nothing gives zeros.  For single tokens and a few at a time; ws: a device tensor as scratch (by default torch's
    allocator is asked)."""
    _, ref, shape, need, device = _paged_plan(q, cache, lam, lengths, scale, causal)
    _current(device)
    out = q.new_empty(shape) if out is None else _given(out, shape, q.dtype, device, "out")
    ws, ptr, nbytes = _ws(ws, need, device)
    rc = _serving_lib().sconv_diffattn_paged(ref, q.data_ptr(), _pages_dev(cache), lam.data_ptr(), lengths.data_ptr(), out.data_ptr(), ptr, nbytes,
                                             _raw_stream(torch))
    if rc:
        raise SconvError(rc, "sconv_diffattn_paged")
    return out
