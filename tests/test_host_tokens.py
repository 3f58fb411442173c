"""The token operators' argument checks: host code that answers before any GPU call."""
import ctypes

import pytest

import paper_1909_09927_amd as sconv
from paper_1909_09927_amd import tokens as T

EINVAL, EUNSUPPORTED = sconv.SCONV_EINVAL, sconv.SCONV_EUNSUPPORTED
P = ctypes.c_void_p(4096)      # never read: every call below is refused or has nothing to do
ODD = ctypes.c_void_p(4100)


def _ln(**kw):
    d = dict(N=2, S=3, C=16, layout=0, x_type=0, y_type=0, w_type=0, eps=1e-5, x_n=48, x_s=16, y_n=48, y_s=16)
    d.update(kw)
    return T.LayerNormDesc(**d)


def _forward(d, x=P, y=P, mean=None, rstd=None):
    return T._tokens_lib().sconv_layernorm_forward(ctypes.byref(d) if d else None, x, None, None, y, mean, rstd, None)


def _backward(d, dy=P, dw=P, db=P, ws=P, nbytes=1 << 30):
    return T._tokens_lib().sconv_layernorm_backward(ctypes.byref(d), dy, P, P, P, None, P, dw, db, ws, nbytes, None)


def test_layernorm_refusals():
    assert _forward(None) == EINVAL
    for bad in (dict(C=0), dict(N=-1), dict(S=-1), dict(layout=2), dict(x_type=2), dict(y_type=-1), dict(w_type=5), dict(eps=-1.0),
                dict(eps=float("inf")), dict(eps=float("nan")), dict(x_type=1, y_type=0), dict(x_s=-1), dict(y_n=-1)):
        assert _forward(_ln(**bad)) == EINVAL, bad
    assert _forward(_ln(C=65537)) == EUNSUPPORTED
    assert _forward(_ln(N=1 << 16, S=1 << 15)) == EUNSUPPORTED
    assert _forward(_ln(), x=None) == EINVAL and _forward(_ln(), y=None) == EINVAL
    assert _forward(_ln(), mean=P) == EINVAL and _forward(_ln(), rstd=P) == EINVAL
    assert _forward(_ln(N=0), x=None, y=None) == 0
    n = ctypes.c_size_t()
    assert T._tokens_lib().sconv_layernorm_workspace_size(ctypes.byref(_ln()), ctypes.byref(n)) == 0 and n.value >= 2 * 16 * 4
    assert T._tokens_lib().sconv_layernorm_workspace_size(ctypes.byref(_ln()), None) == EINVAL
    assert _backward(_ln(), dw=None) == EINVAL and _backward(_ln(), db=None) == EINVAL
    assert _backward(_ln(), nbytes=n.value - 16) == EINVAL and _backward(_ln(), ws=None) == EINVAL
    assert _backward(_ln(), ws=ODD) == EINVAL and _backward(_ln(), dy=None) == EINVAL


def _rotary(q=P, k=P, pos=P, **kw):
    d = dict(B=2, S=3, Hq=2, Hk=1, D=16, type=0, pairs=8, axes=2, interleaved=0, inverse=0)
    d.update({n: v for n, v in kw.items() if n != "axis"})
    desc = T.RotaryDesc(**d)
    axis = kw.get("axis", bytes([0] * 4 + [1] * 4))
    ctypes.memmove(ctypes.addressof(desc) + T.RotaryDesc.axis.offset, axis, len(axis))
    return T._tokens_lib().sconv_rotary(ctypes.byref(desc), q, k, pos, P, P, P, None)


def test_rotary_refusals():
    for bad in (dict(B=-1), dict(S=-1), dict(Hq=-1), dict(Hk=-1), dict(D=0), dict(type=2), dict(pairs=0), dict(pairs=9), dict(axes=0), dict(q_s=-1),
                dict(ko_h=-1), dict(pos_b=-1), dict(axis=bytes([0] * 7 + [2])), dict(q=None), dict(k=None), dict(pos=None)):
        assert _rotary(**bad) == EINVAL, bad
    for big in (dict(D=1026), dict(D=1024, pairs=257), dict(axes=9), dict(B=1 << 16, S=1 << 15), dict(Hq=1 << 20)):
        assert _rotary(**big) == EUNSUPPORTED, big
    assert _rotary(B=0, q=None, k=None, pos=None) == 0
    assert sconv.sconv_rotary_axes((2, 0, 3)) == bytes([0, 0, 2, 2, 2])
    with pytest.raises(ValueError):
        sconv.sconv_rotary_axes((2, -1))


def _attn(**kw):
    d = dict(B=2, Sq=3, Sk=5, H=4, Hkv=2, D=16, Dv=32, type=0, causal=0, scale=0.25)
    d.update(kw)
    return T.DiffAttnDesc(**d)


def _attn_forward(d, q=P, k=P, v=P, lam=P, out=P, second=None, lse=None, ws=None, nbytes=0):
    return T._tokens_lib().sconv_diffattn_forward(ctypes.byref(d) if d else None, q, k, v, lam, None, None, out, second, lse,
                                                  ws, nbytes, None)


def _attn_backward(d, dout=P, k=P, dv=P, dlam=P, ws=P, nbytes=1 << 30):
    return T._tokens_lib().sconv_diffattn_backward(ctypes.byref(d), dout, P, k, P, P, None, None, P, P, P, P, P, dv, dlam, ws,
                                                   nbytes, None)


def test_attention_refusals():
    assert _attn_forward(None) == EINVAL
    for bad in (dict(B=-1), dict(Sq=-1), dict(Sk=-1), dict(H=0), dict(Hkv=0), dict(H=3), dict(D=0), dict(Dv=0), dict(type=2), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_b=-1), dict(k_h=-1), dict(v_s=-1), dict(mask_b=-1)):
        assert _attn_forward(_attn(**bad)) == EINVAL, bad
    for big in (dict(D=129), dict(Dv=257), dict(Sq=(1 << 30) + 1), dict(Sk=(1 << 30) + 1), dict(B=1 << 30, Hkv=2), dict(Sq=1 << 29, H=8)):
        assert _attn_forward(_attn(**big)) == EUNSUPPORTED, big
    for missing in (dict(q=None), dict(k=None), dict(v=None), dict(lam=None), dict(out=None), dict(second=P), dict(lse=P), dict(ws=P),
                    dict(nbytes=64), dict(ws=ODD, nbytes=64)):
        assert _attn_forward(_attn(), **missing) == EINVAL, missing
    assert _attn_forward(_attn(B=0), q=None, k=None, v=None, out=None) == 0
    n = ctypes.c_size_t()
    size = T._tokens_lib().sconv_diffattn_workspace_size
    assert size(ctypes.byref(_attn()), 1, ctypes.byref(n)) == 0 and n.value == 2 * 3 * 4 * 3 * 4
    need = n.value
    assert size(ctypes.byref(_attn()), 0, None) == EINVAL
    for empty in (dict(B=0), dict(Sq=0), dict(Sk=0), dict(B=0, Sq=0, Sk=0)):
        assert size(ctypes.byref(_attn(**empty)), 0, ctypes.byref(n)) == 0 and n.value == 0, empty
    assert size(ctypes.byref(_attn(Sq=1, Sk=4096)), 0, ctypes.byref(n)) == 0 and n.value > 0
    for missing in (dict(dout=None), dict(k=None), dict(dv=None), dict(dlam=None), dict(ws=None), dict(nbytes=need - 4), dict(ws=ODD)):
        assert _attn_backward(_attn(), **missing) == EINVAL, missing


def test_device_tensors_are_asked_for():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4)
    with pytest.raises(TypeError):
        sconv.sconv_layernorm_forward(x)
    with pytest.raises(TypeError):
        sconv.sconv_rotary_forward(torch.zeros(1, 1, 1, 4), None, torch.zeros(1, 1, 1, dtype=torch.int32), torch.ones(2), bytes(2))
    with pytest.raises(AttributeError):
        sconv.sconv_no_such_call


def test_grids_of_2_to_32_threads_are_refused_before_a_launch():
    for big in (dict(N=1, S=1 << 28), dict(N=1, S=1 << 24, C=9000), dict(N=1, S=1 << 24, C=2100, layout=1, x_s=1 << 24),
                dict(N=1 << 21, S=128, C=8, layout=1, x_s=128)):
        assert _forward(_ln(**big)) == EUNSUPPORTED, big
    for big in (dict(N=1, S=1 << 24, C=9000), dict(N=1, S=1 << 24, C=2100, layout=1, x_s=1 << 24)):
        assert _backward(_ln(**big)) == EUNSUPPORTED, big
    assert _rotary(B=1 << 12, S=1 << 12, Hq=64, D=1024) == EUNSUPPORTED
    assert _attn_forward(_attn(B=1 << 24, Sq=1, H=1, Hkv=1)) == EUNSUPPORTED
    assert _attn_forward(_attn(B=1 << 10, Sq=1 << 21, H=1, Hkv=1)) == EUNSUPPORTED
    for big in (dict(B=1, Sq=1 << 28, H=1, Hkv=1), dict(B=1 << 14, Sq=1, Sk=1 << 17, H=1, Hkv=1), dict(B=1, Sq=1, H=1 << 22, Hkv=1)):
        assert _attn_backward(_attn(**big), nbytes=1 << 45) == EUNSUPPORTED, big
