"""The serving operators' argument checks (host code that answers before any GPU call), and their references against closed forms."""
import ctypes
import os
import sys

import numpy as np
import pytest

import paper_1909_09927_amd as sconv

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import serving_ref as ref  # noqa: E402
from paper_1909_09927_amd import serving as S  # noqa: E402

EINVAL, EUNSUPPORTED = sconv.SCONV_EINVAL, sconv.SCONV_EUNSUPPORTED
P = ctypes.c_void_p(4096)      # never read: every call below is refused or has nothing to do
ODD = ctypes.c_void_p(4100)
BY = ctypes.byref


def _rms(**kw):
    d = dict(rows=3, C=16, x_type=0, t_type=0, y_type=0, w_type=0, eps=1e-6, x_r=16, res_r=16, t_r=16, y_r=16)
    d.update(kw)
    return S.RmsNormDesc(**d)


def _rms_forward(d, x=P, res=None, y=P, scale=None, total=None):
    return S._serving_lib().sconv_rmsnorm_forward(BY(d) if d else None, x, res, None, y, scale, total, None, None)


def _rms_backward(d, dy=P, total=P, rstd=P, dw=P, ws=P, nbytes=1 << 30):
    return S._serving_lib().sconv_rmsnorm_backward(BY(d), dy, total, rstd, None, None, P, None, dw, ws, nbytes, None)


def test_rmsnorm_refusals():
    assert _rms_forward(None) == EINVAL
    for bad in (dict(rows=-1), dict(C=0), dict(x_type=2), dict(x_type=-1), dict(t_type=1), dict(t_type=2), dict(y_type=3), dict(x_type=1, t_type=1, y_type=0),
                dict(w_type=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_r=-1), dict(res_r=-1), dict(t_r=-1), dict(y_r=-1)):
        assert _rms_forward(_rms(**bad)) == EINVAL, bad
    for big in (dict(C=16385), dict(rows=(1 << 30) + 1), dict(rows=1 << 28, C=2048)):
        assert _rms_forward(_rms(**big)) == EUNSUPPORTED, big
    for missing in (dict(x=None), dict(y=None), dict(scale=P), dict(res=P), dict(total=P)):
        assert _rms_forward(_rms(), **missing) == EINVAL, missing
    assert _rms_forward(_rms(y_type=2)) == EINVAL
    assert _rms_forward(_rms(rows=0), x=None, y=None) == 0
    n = ctypes.c_size_t()
    assert S._serving_lib().sconv_rmsnorm_workspace_size(BY(_rms()), BY(n)) == 0 and n.value >= 16 * 4
    assert S._serving_lib().sconv_rmsnorm_workspace_size(BY(_rms()), None) == EINVAL
    for missing in (dict(dy=None), dict(total=None), dict(rstd=None), dict(ws=None), dict(ws=ODD), dict(nbytes=n.value - 4)):
        assert _rms_backward(_rms(), **missing) == EINVAL, missing
    assert _rms_backward(_rms(y_type=2)) == EINVAL


def test_quant8_refusals():
    def call(x=P, q=P, s=P, **kw):
        d = dict(M=3, K=200, type=0, block_rows=1, x_m=200, q_m=200)
        d.update(kw)
        return S._serving_lib().sconv_quant8(BY(S.Quant8Desc(**d)), x, q, s, None)

    assert S._serving_lib().sconv_quant8(None, P, P, P, None) == EINVAL
    for bad in (dict(M=-1), dict(K=-1), dict(type=2), dict(block_rows=2), dict(block_rows=0), dict(x_m=-1), dict(q_m=-1), dict(x=None), dict(q=None), dict(s=None)):
        assert call(**bad) == EINVAL, bad
    for big in (dict(M=(1 << 30) + 1), dict(K=(1 << 30) + 1), dict(M=1 << 30, K=1024), dict(M=1 << 30, K=1 << 16, block_rows=128)):
        assert call(**big) == EUNSUPPORTED, big
    assert call(M=0, x=None, q=None, s=None) == 0 and call(K=0, x=None, q=None, s=None) == 0


def test_linear8_refusals():
    def call(x=P, xs=P, w=P, ws=P, y=P, **kw):
        d = dict(M=3, N=5, K=200, y_type=1, x_m=200, w_n=200, y_m=5)
        d.update(kw)
        return S._serving_lib().sconv_linear8(BY(S.Linear8Desc(**d)), x, xs, w, ws, y, None)

    assert S._serving_lib().sconv_linear8(None, P, P, P, P, P, None) == EINVAL
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(y_type=2), dict(x_m=-1), dict(w_n=-1), dict(y_m=-1), dict(x=None), dict(xs=None), dict(w=None),
                dict(ws=None), dict(y=None), dict(K=0, y=None)):
        assert call(**bad) == EINVAL, bad
    for big in (dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 1), dict(K=(1 << 30) + 1), dict(M=1 << 30, N=1 << 30)):
        assert call(**big) == EUNSUPPORTED, big
    assert call(M=0, x=None, y=None) == 0 and call(N=0, w=None, y=None) == 0


def _pages(**kw):
    d = dict(pages=4, page_size=16, table_width=3, type=2, Hk=4, D=16, Hv=2, Dv=32)
    d.update(kw)
    return S.PagesDesc(**d)


def _dev(**kw):
    d = dict(k=4096, v=4096, ks=4096, vs=4096, table=4096)
    d.update(kw)
    return BY(S.PagesDev(**d))


BAD_PAGES = (dict(pages=-1), dict(page_size=0), dict(table_width=-1), dict(type=3), dict(type=1), dict(Hk=0), dict(D=0), dict(Hv=0), dict(Dv=0), dict(k_p=-1), dict(v_h=-1),
             dict(ks_s=-1), dict(vs_p=-1), dict(table_b=-1))
BIG_PAGES = (dict(D=257), dict(Dv=257), dict(table_width=1 << 16, page_size=1 << 15))


def test_cache_refusals():
    L = S._serving_lib()

    def call(k=P, v=P, starts=P, dev=None, pages=None, **kw):
        d = dict(B=2, S=3, type=0)
        d.update(kw)
        desc = BY(S.CacheDesc(**d, pages=_pages(**(pages or {}))))
        dev = _dev() if dev is None else dev
        a, b = L.sconv_cache_write(desc, k, v, starts, None, dev, None), L.sconv_cache_read(desc, dev, starts, None, k, v, None)
        assert a == b
        return a

    assert L.sconv_cache_write(None, P, P, P, None, _dev(), None) == EINVAL
    for bad in (dict(B=-1), dict(S=-1), dict(type=2), dict(k_b=-1), dict(v_s=-1), dict(k=None), dict(v=None), dict(starts=None)):
        assert call(**bad) == EINVAL, bad
    for bad in BAD_PAGES:
        assert call(pages=bad) == EINVAL, bad
    for big in BIG_PAGES:
        assert call(pages=big) == EUNSUPPORTED, big
    assert call(B=1 << 15, S=1 << 15) == EUNSUPPORTED
    for missing in (dict(k=0), dict(v=0), dict(ks=0), dict(vs=0), dict(table=0)):
        assert call(dev=_dev(**missing)) == EINVAL, missing
    assert call(pages=dict(type=0)) == EINVAL                          # (scales without 8 bits)
    assert L.sconv_cache_write(BY(S.CacheDesc(B=2, S=3, type=0, pages=_pages())), P, P, P, None, None, None) == EINVAL
    assert call(B=0, k=None, v=None, starts=None) == 0 and call(S=0, k=None, v=None, starts=None) == 0
    # a cache without pages, or a table without entries: nothing to write
    none = S.CacheDesc(B=2, S=3, type=0, pages=_pages(pages=0))
    assert L.sconv_cache_write(BY(none), P, P, P, None, _dev(k=0, v=0, ks=0, vs=0), None) == 0
    none = S.CacheDesc(B=2, S=3, type=0, pages=_pages(table_width=0))
    assert L.sconv_cache_write(BY(none), P, P, P, None, _dev(table=0), None) == 0


def test_paged_refusals():
    L = S._serving_lib()

    def call(q=P, dev=None, lam=P, lengths=P, out=P, ws=None, nbytes=0, pages=None, **kw):
        d = dict(B=2, Sq=3, H=4, Hkv=2, type=0, causal=0, scale=0.25)
        d.update(kw)
        desc = S.PagedDesc(**d, pages=_pages(**(pages or {})))
        return L.sconv_diffattn_paged(BY(desc), q, _dev() if dev is None else dev, lam, lengths, out, ws, nbytes, None)

    assert L.sconv_diffattn_paged(None, P, _dev(), P, P, P, None, 0, None) == EINVAL
    for bad in (dict(B=-1), dict(Sq=-1), dict(H=0), dict(Hkv=0), dict(H=3), dict(type=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(q_b=-1), dict(q_s=-1), dict(q_h=-1), dict(Hkv=1), dict(pages=dict(Hv=3)), dict(pages=dict(Hk=3)), dict(q=None),
                dict(lam=None), dict(lengths=None), dict(out=None), dict(ws=P), dict(nbytes=64), dict(ws=ODD, nbytes=64)):
        assert call(**bad) == EINVAL, bad
    for bad in BAD_PAGES:
        assert call(pages=bad) == EINVAL, bad
    for big in BIG_PAGES + (dict(D=129),):
        assert call(pages=big) == EUNSUPPORTED, big
    for big in (dict(Sq=(1 << 20) + 1), dict(B=(1 << 24) + 1), dict(H=1 << 21), dict(B=1 << 12, Sq=1 << 12)):
        assert call(**big) == EUNSUPPORTED, big
    for missing in (dict(k=0), dict(v=0), dict(ks=0), dict(vs=0), dict(table=0)):
        assert call(dev=_dev(**missing)) == EINVAL, missing
    assert call(pages=dict(type=0)) == EINVAL
    assert call(B=0, q=None, out=None) == 0 and call(Sq=0, q=None, out=None) == 0
    n = ctypes.c_size_t()
    size = L.sconv_diffattn_paged_workspace_size
    assert size(BY(S.PagedDesc(B=2, Sq=1, H=4, Hkv=2, type=0, scale=1.0, pages=_pages(table_width=300))), BY(n)) == 0 and n.value > 0
    for empty in (dict(Sq=0), dict(B=0), dict(Sq=0, B=0), dict(pages=_pages(table_width=0)), dict(pages=_pages(pages=0, table_width=0))):
        assert size(BY(S.PagedDesc(**{**dict(B=2, Sq=1, H=4, Hkv=2, type=0, scale=1.0, pages=_pages()), **empty})), BY(n)) == 0 and n.value == 0, empty
    assert size(BY(S.PagedDesc(B=2, Sq=1, H=4, Hkv=2, type=0, scale=1.0, pages=_pages())), None) == EINVAL
    # many rows: as many wavefronts as the chip has places for without parts, which would take 272 MB
    assert size(BY(S.PagedDesc(B=2, Sq=1024, H=128, Hkv=2, type=0, scale=1.0, pages=_pages(table_width=300))), BY(n)) == 0 and n.value == 0


def test_device_tensors_are_asked_for():
    x = torch.zeros(2, 4)
    cache = sconv.sconv_cache_new(1, 2, 3, 4, 2, 8, 1, 8, device="cpu")
    assert cache.k.shape == (3, 4, 2, 8) and cache.v_scales.shape == (3, 4, 1) and cache.table.tolist() == [[-1, -1]]
    assert sconv.sconv_cache_new(1, 2, 3, 4, 2, 8, 1, 8, dtype=torch.bfloat16, device="cpu").k_scales is None
    one = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: sconv.sconv_rmsnorm_forward(x), lambda: sconv.sconv_rmsnorm_backward(x, x, x), lambda: sconv.sconv_quant8(x),
                 lambda: sconv.sconv_linear8((x, x), (x, x)), lambda: sconv.sconv_cache_write(cache, x, x, one), lambda: sconv.sconv_cache_read(cache, 1, one),
                 lambda: sconv.sconv_diffattn_paged(x, cache, x, one), lambda: sconv.sconv_rmsnorm_forward(None)):
        with pytest.raises(TypeError):
            call()


def test_reference_scales_and_bytes():
    """The references' 8-bit values against torch's own conversion, their scales against the definition at its borders."""
    f = np.array([0.0, 448.0, 448.0000001, 449.0, 896.0, 896.1, 1.75, 1.7500001, 3.4028234663852886e38, 2.0 ** -149, 448.0 * 2.0 ** -126, 450.0 * 2.0 ** -126])
    assert ref.scale_byte(f).tolist() == [1, 127, 128, 128, 128, 129, 119, 120, 247, 1, 1, 2]
    g = torch.Generator()
    g.manual_seed(0)
    x = torch.cat([torch.randn(4096, generator=g) * 100, torch.randn(4096, generator=g) * 1e-2, torch.linspace(-448, 448, 4001)]).clamp(-448, 448)
    assert (ref._to8(x.double().numpy()) == x.to(ref.E4M3).view(torch.uint8).numpy()).all()
    assert np.array_equal(ref.VALUES8, torch.arange(256, dtype=torch.uint8).view(ref.E4M3).double().numpy(), equal_nan=True)


def test_division_by_multiplication():
    """The page division's constants: exact at every multiple and its neighbours."""
    rng = np.random.RandomState(0)
    for d in [1, 2, 3, 7, 16, 20, 24, 63, 64, 100, 641, 65535, 65537, (1 << 30) + 1, (1 << 31) - 1] + rng.randint(1, 1 << 31, 200).tolist():
        l = 0
        while (1 << l) < d:
            l += 1
        m = ((1 << (31 + l)) + d - 1) // d
        assert m < 1 << 32
        top = (1 << 31) - 1
        for q in [0, 1, 2, top // d] + rng.randint(0, top // d + 1, 20).tolist():
            for n in (q * d - 1, q * d, q * d + d - 1, top):
                if 0 <= n <= top:
                    assert n * m >> (31 + l) == n // d
