"""The token operators against plain implementations in 64 bits (tokens_ref), at the sizes, strides and masks where they can
go wrong.  Bounds come from the inputs and the types (tokens_ref)."""
import math

import pytest
import torch

import paper_1909_09927_amd as sconv
import tokens_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g).to(dtype)


# ---- layer norm

NORM_SHAPES = [(1, 1, 1), (1, 1, 16), (2, 3, 17), (3, 5, 30), (1, 49, 2048), (2, 700, 64), (1, 1500, 128), (2, 33, 256), (4, 300, 257),
               (1, 70, 700), (2, 600, 1024), (1, 1030, 2048), (1, 9, 2050), (1, 40, 4096), (1, 5, 5001), (1, 3, 8192), (2, 2, 9000)]
TYPES = [(F32, F32), (BF16, BF16), (F32, BF16)]


@pytest.mark.parametrize("types", TYPES, ids=["fp32", "bf16", "fp32-bf16"])
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=str)
def test_norm_tokens(device, shape, types):
    g = _gen(sum(shape))
    N, S, C = shape
    x = (_randn(g, N, S, C) * 1.7 + 3.0).to(types[0])
    w, b = 1.0 + 0.2 * _randn(g, C), _randn(g, C)
    dy = _randn(g, N, S, C, dtype=types[1])
    y, mean, rstd = sconv.sconv_layernorm_forward(x.to(device), w.to(device), b.to(device), out_dtype=types[1], stats=True)
    (ry, rm, rr), (by, bm, br) = ref.norm(x, w, b, 1e-5, types[1])
    ref.within(y, ry, by, "y")
    ref.within(mean, rm, bm, "mean")
    ref.within(rstd, rr, br, "rstd")
    dx, dw, db = sconv.sconv_layernorm_backward(dy.to(device), x.to(device), mean, rstd, w.to(device))
    (rx, rw, rb), (bx, bw, bb) = ref.norm_grad(dy, x, mean.cpu(), rstd.cpu(), w)
    ref.within(dx, rx, bx + 1.01 * ref.U[types[0]] * rx.abs(), "dx")
    ref.within(dw, rw, bw + 2 * ref.E * rw.abs(), "dweight")
    ref.within(db, rb, bb + 2 * ref.E * rb.abs(), "dbias")


MAP_SHAPES = [(1, 1, 1, 1), (2, 17, 3, 5), (1, 64, 7, 7), (3, 128, 5, 9), (2, 130, 8, 8), (1, 256, 14, 14), (2, 300, 6, 11), (1, 513, 4, 4),
              (1, 896, 14, 14), (1, 1024, 3, 11), (1, 1500, 5, 5), (2, 2048, 7, 7), (1, 2100, 3, 3)]


@pytest.mark.parametrize("types", TYPES, ids=["fp32", "bf16", "fp32-bf16"])
@pytest.mark.parametrize("shape", MAP_SHAPES, ids=str)
def test_norm_map(device, shape, types):
    g = _gen(sum(shape))
    N, C, H, W = shape
    x = (_randn(g, N, C, H, W) + 0.3).relu().to(types[0])
    w, b = 1.0 + 0.2 * _randn(g, C), _randn(g, C)
    dy = _randn(g, N, H * W, C, dtype=types[1])
    y, mean, rstd = sconv.sconv_layernorm_forward(x.to(device), w.to(device), b.to(device), layout="map",
                                                  out_dtype=types[1], stats=True)
    tokens = x.flatten(2).transpose(1, 2)
    (ry, rm, rr), (by, bm, br) = ref.norm(tokens, w, b, 1e-5, types[1])
    ref.within(y, ry, by, "y")
    ref.within(mean, rm, bm, "mean")
    ref.within(rstd, rr, br, "rstd")
    dx, dw, db = sconv.sconv_layernorm_backward(dy.to(device), x.to(device), mean, rstd, w.to(device), layout="map")
    assert dx.shape == x.shape and dx.is_contiguous()
    (rx, rw, rb), (bx, bw, bb) = ref.norm_grad(dy, tokens, mean.cpu(), rstd.cpu(), w)
    ref.within(dx.flatten(2).transpose(1, 2), rx, bx + 1.01 * ref.U[types[0]] * rx.abs(), "dx")
    ref.within(dw, rw, bw + 2 * ref.E * rw.abs(), "dweight")
    ref.within(db, rb, bb + 2 * ref.E * rb.abs(), "dbias")


@pytest.mark.parametrize("types", TYPES, ids=["fp32", "bf16", "fp32-bf16"])
@pytest.mark.parametrize("shape", [(300, 70, 1, 5), (48, 200, 14, 14), (20, 300, 14, 15), (64, 520, 5, 13)], ids=str)
def test_norm_map_of_many_tiles(device, shape, types):
    """More tiles than compute units, and than rows of partial sums."""
    test_norm_map(device, shape, types)


@pytest.mark.parametrize("layout", ["tokens", "map"])
def test_norm_plain_and_weight_types(device, layout):
    g = _gen(5)
    N, S, C = 3, 40, 72
    x = _randn(g, N, S, C) if layout == "tokens" else _randn(g, N, C, S)
    rows = x if layout == "tokens" else x.transpose(1, 2)
    xd = x.to(device)
    dy = _randn(g, N, S, C)
    for w, b in ((None, None), (_randn(g, C), None), (None, _randn(g, C)), (_randn(g, C, dtype=BF16), _randn(g, C, dtype=BF16))):
        dev = [None if t is None else t.to(device) for t in (w, b)]
        y, mean, rstd = sconv.sconv_layernorm_forward(xd, *dev, eps=1e-3, layout=layout, stats=True)
        (ry, _, _), (by, _, _) = ref.norm(rows, w, b, 1e-3, F32)
        ref.within(y, ry, by, "y")
        assert torch.equal(y, sconv.sconv_layernorm_forward(xd, *dev, eps=1e-3, layout=layout))
        dx, dw, db = sconv.sconv_layernorm_backward(dy.to(device), xd, mean, rstd, dev[0], layout=layout)
        (rx, rw, rb), (bx, bw, bb) = ref.norm_grad(dy, rows, mean.cpu(), rstd.cpu(), w)
        dx = dx if layout == "tokens" else dx.transpose(1, 2)
        ref.within(dx, rx, bx + 2 * ref.E * rx.abs(), "dx")
        t = F32 if w is None else w.dtype
        assert dw.dtype == db.dtype == t
        ref.within(dw, rw, bw + 1.01 * ref.U[t] * rw.abs(), "dweight")
        ref.within(db, rb, bb + 1.01 * ref.U[t] * rb.abs(), "dbias")
        only, none, none2 = sconv.sconv_layernorm_backward(dy.to(device), xd, mean, rstd, dev[0], layout=layout, param_grads=False)
        assert none is None and none2 is None and torch.equal(only if layout == "tokens" else only.transpose(1, 2), dx)


@pytest.mark.parametrize("C", [64, 96, 513])
def test_norm_strides(device, C):
    """Slices of a wider tensor, broadcast images, heads of a token, a padded map."""
    g = _gen(6)
    wide = _randn(g, 4, 21, C + 40).to(device)
    for x in (wide[:, :, 8:8 + C], wide[:, 3:20, 5:5 + C], wide[1:2, :, :C].expand(4, 21, C)):
        y, mean, rstd = sconv.sconv_layernorm_forward(x, stats=True)
        (ry, _, _), (by, _, _) = ref.norm(x.cpu(), None, None, 1e-5, F32)
        ref.within(y, ry, by, "y")
        dy = torch.randn(x.shape[0], x.shape[1], C + 8, device=device)[:, :, 8:]
        dx, dw, db = sconv.sconv_layernorm_backward(dy, x, mean, rstd)
        (rx, rw, rb), (bx, bw, bb) = ref.norm_grad(dy.cpu(), x.cpu(), mean.cpu(), rstd.cpu(), None)
        ref.within(dx, rx, bx + 2 * ref.E * rx.abs(), "dx")
        ref.within(dw, rw, bw + 2 * ref.E * rw.abs(), "dweight")
    heads = _randn(g, 2, 5, 4, C).to(device)
    (ry, _, _), (by, _, _) = ref.norm(heads.cpu(), None, None, 1e-5, F32)
    ref.within(sconv.sconv_layernorm_forward(heads), ry, by, "heads")
    maps = _randn(g, 3, C + 6, 5, 7).to(device)[:, 3:3 + C]
    (ry, _, _), (by, _, _) = ref.norm(maps.cpu().flatten(2).transpose(1, 2), None, None, 1e-5, F32)
    ref.within(sconv.sconv_layernorm_forward(maps, layout="map"), ry, by, "map")


def test_norm_rows_stand_alone_and_large_mean(device):
    g = _gen(7)
    x = _randn(g, 6, 300) + 3000.0
    x[2, 5] = float("nan")
    x[4, 7] = float("inf")
    y = sconv.sconv_layernorm_forward(x.to(device)).cpu()
    keep = [0, 1, 3, 5]
    (ry, _, _), (by, _, _) = ref.norm(x[keep], None, None, 1e-5, F32)
    ref.within(y[keep], ry, by, "y")
    assert y[2].isnan().all() and y[4].isnan().any()
    for layout, shape in (("tokens", (0, 5, 8)), ("tokens", (2, 0, 8)), ("map", (0, 8, 2, 2))):
        x = torch.empty(shape, device=device)
        y, mean, rstd = sconv.sconv_layernorm_forward(x, layout=layout, stats=True)
        dx, dw, db = sconv.sconv_layernorm_backward(y, x, mean, rstd, layout=layout)
        assert y.numel() == dx.numel() == 0 and not dw.any() and not db.any()


def _differences(f, args, grads, seed, step=1e-5):
    """The gradients along random directions against central differences of f in 64 bits."""
    g = _gen(seed)
    for k, (a, d) in enumerate(zip(args, grads)):
        v = torch.randn(a.shape, generator=g, dtype=torch.float64)
        up, down = ([t + s * step * v if i == k else t for i, t in enumerate(args)] for s in (1, -1))
        want = (f(*up) - f(*down)) / (2 * step)
        got = (d.double().cpu() * v).sum()
        # fp32 gradients: each within a few 2^-24 of its scale, summed over random signs; differences: step^2
        tol = 1e-5 * float((d.double().cpu().norm() * v.norm())) + 1e-6
        assert abs(float(got - want)) <= tol, (k, float(got), float(want), tol)


def test_norm_gradient_against_differences(device):
    g = _gen(8)
    x, w, b, dy = _randn(g, 5, 33), 1.0 + 0.2 * _randn(g, 33), _randn(g, 33), _randn(g, 5, 33)
    y, mean, rstd = sconv.sconv_layernorm_forward(x.to(device), w.to(device), b.to(device), stats=True)
    grads = sconv.sconv_layernorm_backward(dy.to(device), x.to(device), mean, rstd, w.to(device))
    _differences(lambda x, w, b: (ref.norm(x, w, b, 1e-5, F32)[0][0] * dy.double()).sum(), [t.double() for t in (x, w, b)], grads, 9)


# ---- rotary positions

@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 2, (1,)), (2, 1, 16, 4, 64, (12, 10, 10)), (3, 17, 4, 2, 32, (8, 8)), (2, 5, 3, 0, 24, (5, 4)),
                                   (1, 300, 2, 1, 128, (16, 24, 24)), (2, 30, 4, 4, 64, (8, 8)), (1, 9, 2, 2, 70, (11, 13, 3, 8)),
                                   (64, 1, 2, 2, 96, (48,)), (1, 40, 5, 1, 7, (2, 1))], ids=str)
def test_rotary(device, shape, interleaved, dtype):
    B, S, Hq, Hk, D, sections = shape
    g = _gen(sum(shape[:5]))
    q, k = _randn(g, B, S, Hq, D, dtype=dtype), _randn(g, B, S, Hk, D, dtype=dtype) if Hk else None
    axes = sconv.sconv_rotary_axes(sections)
    freq = torch.tensor([10000.0 ** (-i / n) for n in sections for i in range(n)])
    for batch in (1, B):
        pos = torch.randint(-100, 5000, (batch, S, len(sections)), generator=g, dtype=torch.int32)
        dev = [None if t is None else t.to(device) for t in (q, k, pos, freq)]
        for call, inverse in ((sconv.sconv_rotary_forward, False), (sconv.sconv_rotary_backward, True)):
            for x, y in zip((q, k), call(*dev, axes, interleaved=interleaved)):
                if x is None:
                    assert y is None
                    continue
                want, bound = ref.rotary(x, pos, freq, axes, interleaved, inverse)
                ref.within(y, want, bound + 1.01 * ref.U[dtype] * want.abs(), "turned")
    kept = [None if t is None else t.clone() for t in dev]
    a = sconv.sconv_rotary_forward(*dev, axes, interleaved=interleaved)
    b = sconv.sconv_rotary_forward(*kept, axes, interleaved=interleaved, out=(kept[0], kept[1]))     # in place
    assert b[0] is kept[0] and torch.equal(a[0], b[0]) and (k is None or torch.equal(a[1], b[1]))


def test_rotary_slices_and_far_places(device):
    g = _gen(11)
    both = _randn(g, 2, 50, 9, 64, dtype=BF16).to(device)
    q, k = both[:, :, 1:5], both[:, :, 5:7]
    axes, freq = sconv.sconv_rotary_axes((16, 16)), torch.tensor([10000.0 ** (-i / 16) for i in range(16)] * 2)
    pos = torch.randint(0, 2 ** 31 - 1, (1, 50, 2), generator=g, dtype=torch.int32)
    for interleaved in (False, True):
        for x, y in zip((q, k), sconv.sconv_rotary_forward(q, k, pos.to(device), freq.to(device), axes, interleaved)):
            want, bound = ref.rotary(x.cpu(), pos, freq, axes, interleaved, False)
            # (2^31 * 2^-53 turns of the angle in 64 bits, on both sides)
            ref.within(y, want, bound + 1e-6 + 1.01 * ref.U[BF16] * want.abs(), "turned")
    odd = torch.randn(2, 50, 4, 65, device=device)[..., 1:]
    want, bound = ref.rotary(odd.cpu(), pos, freq, axes, False, False)
    y, _ = sconv.sconv_rotary_forward(odd, None, pos.to(device), freq.to(device), axes)
    ref.within(y, want, bound + 1e-6 + 2 * ref.E * want.abs(), "turned")
    e = torch.empty(0, 3, 2, 64, device=device)
    assert sconv.sconv_rotary_forward(e, e, pos[:, :3].contiguous().to(device), freq.to(device), axes)[0].shape == e.shape


# ---- differential attention

def _attention_inputs(g, B, Sq, Sk, H, Hkv, D, Dv, dtype, spread=1.5):
    return ((spread * _randn(g, B, Sq, 2 * H, D)).to(dtype), _randn(g, B, Sk, 2 * Hkv, D, dtype=dtype),
            _randn(g, B, Sk, Hkv, Dv, dtype=dtype), 0.5 + 0.2 * _randn(g, H), _randn(g, B, Sq, H, Dv, dtype=dtype))


def _attention_check(device, q, k, v, lam, dout, scale=None, causal=False, lengths=None, mask=None, grad=True):
    r, e = ref.attention(q, k, v, lam, scale, causal, lengths, mask, dout if grad else None)
    d = [t if t.is_cuda else t.to(device) for t in (q, k, v, lam, dout)]
    kw = dict(scale=scale, causal=causal, k_lengths=None if lengths is None else lengths.to(device),
              k_mask=None if mask is None else mask.to(device))
    out, second, lse = sconv.sconv_diffattn_forward(*d[:4], save=True, **kw)
    for name, got in (("out", out), ("second", second), ("lse", lse)):
        ref.within(got, r[name], e[name], name)
    assert torch.equal(out, sconv.sconv_diffattn_forward(*d[:4], **kw))
    if grad:
        got = sconv.sconv_diffattn_backward(d[4], *d[:4], out, second, lse, **kw)
        for name, t in zip(("dq", "dk", "dv", "dlam"), got):
            ref.within(t, r[name], e[name], name)
        for a, b in zip(got, sconv.sconv_diffattn_backward(d[4], *d[:4], out, second, lse, **kw)):
            assert torch.equal(a, b)
    return out


ATTENTION = [  # B, Sq, Sk, H, Hkv, D, Dv
    (1, 1, 1, 1, 1, 64, 128), (2, 5, 7, 2, 1, 32, 64), (1, 33, 65, 1, 1, 16, 32), (1, 130, 130, 2, 2, 64, 128), (2, 49, 49, 7, 7, 64, 128),
    (1, 64, 200, 4, 2, 64, 64), (1, 31, 129, 3, 1, 24, 48), (1, 40, 40, 2, 1, 128, 256), (1, 35, 70, 1, 1, 100, 37), (2, 20, 50, 2, 2, 13, 27),
    (1, 70, 33, 2, 1, 72, 144), (1, 9, 100, 2, 2, 20, 200)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", ATTENTION, ids=str)
def test_attention(device, shape, causal, dtype):
    _attention_check(device, *_attention_inputs(_gen(sum(shape)), *shape, dtype), causal=causal)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_lengths_and_masks(device, causal, dtype):
    """Lengths of zero, one, across tiles and (to be cut) beyond the cache; masks that leave rows and whole requests empty."""
    g = _gen(21)
    lengths = torch.tensor([0, 1, 32, 33, 100, 97, 1000, -3], dtype=torch.int32)
    q, k, v, lam, dout = _attention_inputs(g, 8, 34, 100, 2, 1, 64, 128, dtype)
    _attention_check(device, q, k, v, lam, dout, causal=causal, lengths=lengths)
    mask = torch.rand(8, 100, generator=g) < 0.6
    mask[1] = False
    mask[2] = False
    mask[2, 99] = True
    mask[4, :64] = False
    _attention_check(device, q, k, v, lam, dout, causal=causal, lengths=lengths, mask=mask)
    _attention_check(device, q, k, v, lam, dout, causal=causal, mask=mask)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_left_out_places_may_hold_anything(device, dtype):
    """Inf, NaN and the type's lowest value in keys and values that lengths or the mask leave out, and in the queries and gradients
    of rows that see nothing."""
    g = _gen(22)
    B, Sq, Sk = 3, 40, 90
    q, k, v, lam, dout = _attention_inputs(g, B, Sq, Sk, 2, 2, 32, 64, dtype)
    lengths = torch.tensor([90, 41, 0], dtype=torch.int32)
    mask = torch.rand(B, Sk, generator=g) < 0.7
    mask[:, 0] = True
    gone = ~ref.visible(B, Sq, Sk, False, lengths, mask)[:, 0]
    clean = _attention_check(device, q, k, v, lam, dout, lengths=lengths, mask=mask)
    for junk in (float("nan"), float("inf"), torch.finfo(dtype).min):
        kj, vj, qj, dj = k.clone(), v.clone(), q.clone(), dout.clone()
        kj[gone], vj[gone], qj[2], dj[2] = junk, junk, junk, junk
        assert torch.equal(clean, _attention_check(device, qj, kj, vj, lam, dj, lengths=lengths, mask=mask))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 1, 700, 4, 1, 64, 128), (2, 1, 3000, 16, 4, 64, 128), (1, 2, 2049, 8, 8, 32, 64), (2, 1, 1500, 3, 1, 128, 256),
                                   (1, 1, 1, 2, 2, 64, 128), (1, 5, 900, 6, 1, 40, 80), (1, 50, 1700, 2, 1, 64, 128)], ids=str)
def test_attention_step(device, shape, dtype):
    """Few queries over a cache: split keys, with and without scratch, requests of very different lengths."""
    g = _gen(sum(shape))
    B, Sq, Sk = shape[:3]
    q, k, v, lam, dout = _attention_inputs(g, *shape, dtype)
    lengths = torch.tensor([Sk, 0, Sk // 3][:B], dtype=torch.int32)
    for n in (None, lengths, torch.clamp(lengths, max=Sq)):
        _attention_check(device, q, k, v, lam, dout, causal=True, lengths=n, grad=False)
    r, e = ref.attention(q, k, v, lam, None, True, lengths, None)
    dev = [t.to(device) for t in (q, k, v, lam)]
    need = sconv.sconv_diffattn_workspace_size(*dev)
    for nbytes in {16, need // 2 // 16 * 16 + 16, need + 64}:
        ws = torch.full((nbytes,), 255, dtype=torch.uint8, device=device)        # NaN in every float
        out = sconv.sconv_diffattn_forward(*dev, causal=True, k_lengths=lengths.to(device), ws=ws)
        ref.within(out, r["out"], e["out"], f"out with {nbytes} bytes of scratch")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_strides(device, dtype):
    """Slices of one projection, a cache with room, broadcast keys, addresses that are not aligned."""
    g = _gen(23)
    B, S, H, Hkv, D, Dv = 2, 45, 4, 2, 32, 64
    for shift in (0, 1):
        row = _randn(g, B, S, 2 * H * D + 2 * Hkv * D + Hkv * Dv + shift, dtype=dtype).to(device)[..., shift:]
        q = row[..., :2 * H * D].unflatten(2, (2 * H, D))
        k = row[..., 2 * H * D:2 * (H + Hkv) * D].unflatten(2, (2 * Hkv, D))
        v = row[..., 2 * (H + Hkv) * D:].unflatten(2, (Hkv, Dv))
        lam, dout = 0.5 + 0.2 * _randn(g, H), _randn(g, B, S, H, Dv, dtype=dtype)
        r, e = ref.attention(q.cpu(), k.cpu(), v.cpu(), lam, None, True, None, None, dout.cpu())
        out, second, lse = sconv.sconv_diffattn_forward(q, k, v, lam.to(device), causal=True, save=True)
        ref.within(out, r["out"], e["out"], "out")
        got = sconv.sconv_diffattn_backward(dout.to(device), q, k, v, lam.to(device), out, second, lse, causal=True)
        for name, t in zip(("dq", "dk", "dv", "dlam"), got):
            ref.within(t, r[name], e[name], name)
    # keys laid out head by head, the cache of one request shared by all
    k = _randn(g, 1, 2 * Hkv, 60, D, dtype=dtype).to(device).transpose(1, 2)[:, :50].expand(B, 50, 2 * Hkv, D)
    v = _randn(g, 1, Hkv, 60, Dv, dtype=dtype).to(device).transpose(1, 2)[:, :50].expand(B, 50, Hkv, Dv)
    r, e = ref.attention(q.cpu(), k.cpu(), v.cpu(), lam, 0.3, False, None, None)
    ref.within(sconv.sconv_diffattn_forward(q, k, v, lam.to(device), scale=0.3), r["out"], e["out"], "out")


def test_attention_cache_past_32_bits(device):
    """A cache whose last request lies beyond 2^32 bytes (and 2^31 elements) from its start."""
    B, Sk, Hkv, D, Dv = 3, 40, 1, 64, 128
    g = _gen(24)
    stride = (1 << 31) + 64                     # elements between requests
    store = torch.empty((B - 1) * stride + Sk * 256, dtype=BF16, device=device)
    k = store.as_strided((B, Sk, 2, D), (stride, 256, D, 1))
    v = store[128:].as_strided((B, Sk, 1, Dv), (stride, 256, Dv, 1))
    q, kk, vv, lam, dout = _attention_inputs(g, B, 3, Sk, 2, Hkv, D, Dv, BF16)
    k.copy_(kk.to(device))
    v.copy_(vv.to(device))
    r, e = ref.attention(q, kk, vv, lam, None, True, None, None)
    ref.within(sconv.sconv_diffattn_forward(q.to(device), k, v, lam.to(device), causal=True), r["out"], e["out"], "out")


def test_attention_extreme_scores(device):
    """Scores far apart (one key takes all), equal ones, very negative ones, and lam of 0 and below it."""
    g = _gen(25)
    q, k, v, lam, dout = _attention_inputs(g, 1, 50, 150, 4, 2, 64, 128, F32, spread=40.0)
    lam[0], lam[1] = 0.0, -1.5
    _attention_check(device, q, k, v, lam, dout)
    _attention_check(device, q * 0.0, k, v, lam, dout)
    _attention_check(device, q.abs(), -k.abs() * 3, v, lam, dout, causal=True)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 300, 520, 4, 1, 64, 128), (2, 150, 300, 6, 2, 32, 64), (1, 200, 300, 4, 2, 128, 256), (1, 260, 260, 8, 1, 74, 148),
                                   (3, 257, 259, 2, 2, 32, 64), (1, 500, 64, 3, 3, 64, 128)], ids=str)
def test_attention_in_parts(device, shape, causal, dtype):
    """Gradients whose keys, or heads and queries, are split over workgroups; tiles that end inside, with lengths, masks and lam of any sign."""
    g = _gen(sum(shape) + 1)
    B, Sq, Sk, H = shape[:4]
    q, k, v, lam, dout = _attention_inputs(g, *shape, dtype)
    lam[0] = -0.7
    lam[-1] = 0.0
    lengths = torch.tensor([Sk - 3, 65, Sk][:B], dtype=torch.int32)
    mask = torch.rand(B, Sk, generator=g) < 0.8
    mask[:, 32:128] = False
    mask[:, 40] = True
    _attention_check(device, q, k, v, lam, dout, causal=causal, lengths=lengths)
    _attention_check(device, q, k, v, lam, dout, causal=causal, lengths=lengths, mask=mask)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("D", [64, 72])
def test_attention_junk_in_whole_tiles(device, D, dtype):
    """Keys that are left out over whole tiles and at a cache's end, holding NaN and Inf, under heads whose tiles go to LDS directly
    (64) and through registers (72)."""
    g = _gen(41 + D)
    B, Sq, Sk = 2, 70, 200
    q, k, v, lam, dout = _attention_inputs(g, B, Sq, Sk, 2, 2, D, 2 * D, dtype)
    lengths = torch.tensor([193, 130], dtype=torch.int32)
    mask = torch.rand(B, Sk, generator=g) < 0.9
    mask[0, 64:128] = False
    for m in (None, mask):
        gone = ~ref.visible(B, Sq, Sk, False, lengths, m)[:, 0]
        clean = _attention_check(device, q, k, v, lam, dout, lengths=lengths, mask=m)
        for junk in (float("nan"), float("inf")):
            kj, vj = k.clone(), v.clone()
            kj[gone], vj[gone] = junk, junk
            assert torch.equal(clean, _attention_check(device, q, kj, vj, lam, dout, lengths=lengths, mask=m))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_keys_head_by_head(device, dtype):
    """Keys and values laid out [B, heads, capacity, D], as a cache of heads is, with NaN in the places beyond the last key: forward,
    backward and single tokens."""
    g = _gen(51)
    B, Sk, H, D = 2, 100, 2, 64
    q, kk, vv, lam, dout = _attention_inputs(g, B, 80, Sk, H, H, D, 2 * D, dtype)
    k = torch.full((B, 2 * H, 130, D), float("nan"), dtype=dtype, device=device).transpose(1, 2)[:, :Sk]
    v = torch.full((B, H, 130, 2 * D), float("nan"), dtype=dtype, device=device).transpose(1, 2)[:, :Sk]
    k.copy_(kk.to(device))
    v.copy_(vv.to(device))
    r, e = ref.attention(q, kk, vv, lam, None, True, None, None, dout)
    dev = q.to(device), k, v, lam.to(device)
    out, second, lse = sconv.sconv_diffattn_forward(*dev, causal=True, save=True)
    ref.within(out, r["out"], e["out"], "out")
    for name, t in zip(("dq", "dk", "dv", "dlam"), sconv.sconv_diffattn_backward(dout.to(device), *dev, out, second, lse, causal=True)):
        ref.within(t, r[name], e[name], name)
    r, e = ref.attention(q[:, -1:], kk, vv, lam, None, True, None, None)
    ref.within(sconv.sconv_diffattn_forward(q[:, -1:].contiguous().to(device), *dev[1:], causal=True), r["out"], e["out"], "one token")


def test_attention_empty_axes(device):
    for B, Sq, Sk in ((0, 3, 4), (2, 0, 4), (2, 3, 0)):
        q, k = torch.randn(B, Sq, 4, 32, device=device), torch.randn(B, Sk, 4, 32, device=device)
        v, lam = torch.randn(B, Sk, 2, 64, device=device), torch.ones(2, device=device)
        out, second, lse = sconv.sconv_diffattn_forward(q, k, v, lam, save=True)
        assert out.shape == (B, Sq, 2, 64) and not out.any() and not second.any() and (lse == -math.inf).all()
        grads = sconv.sconv_diffattn_backward(torch.randn_like(out), q, k, v, lam, out, second, lse)
        assert all(not t.any() for t in grads)


def test_attention_gradient_against_differences(device):
    g = _gen(26)
    q, k, v, lam, dout = _attention_inputs(g, 2, 11, 19, 4, 2, 16, 24, F32)
    dev = [t.to(device) for t in (q, k, v, lam)]
    out, second, lse = sconv.sconv_diffattn_forward(*dev, causal=True, save=True)
    grads = sconv.sconv_diffattn_backward(dout.to(device), *dev, out, second, lse, causal=True)

    def f(q, k, v, lam):
        seen = ref.visible(2, 11, 19, True, None, None)
        total = 0.0
        for h in range(4):
            a = [torch.softmax((q[:, :, 2 * h + m] @ k[:, :, 2 * (h // 2) + m].transpose(1, 2) / 4.0).masked_fill(~seen, -math.inf), 2)
                 for m in (0, 1)]
            total = total + (((a[0] - lam[h] * a[1]) @ v[:, :, h // 2]) * dout[:, :, h].double()).sum()
        return total

    _differences(f, [t.double() for t in (q, k, v, lam)], grads, 27)


# ---- streams, graphs, refusals

def test_tokens_on_another_stream_and_in_a_graph(device):
    g = _gen(31)
    x = _randn(g, 2, 64, 6, 6).to(device)
    w = torch.ones(64, device=device)
    lam = torch.full((2,), 0.4, device=device)
    axes, freq = sconv.sconv_rotary_axes((4, 4)), torch.tensor([1.0, 0.1, 0.01, 0.001] * 2, device=device)
    pos = torch.cartesian_prod(torch.arange(6), torch.arange(6)).to(torch.int32).to(device)

    def step():
        t, mean, rstd = sconv.sconv_layernorm_forward(x, w, None, layout="map", out_dtype=BF16, stats=True)
        q, k = sconv.sconv_rotary_forward(t.unflatten(2, (4, 16)), t.unflatten(2, (4, 16)), pos, freq, axes)
        v = t.unflatten(2, (2, 32))
        out, second, lse = sconv.sconv_diffattn_forward(q, k, v, lam, causal=True, save=True)
        one = sconv.sconv_diffattn_forward(q[:, -1:].contiguous(), k, v, lam)
        grads = sconv.sconv_diffattn_backward(out, q, k, v, lam, out, second, lse, causal=True)
        dx, dw, db = sconv.sconv_layernorm_backward(grads[2].flatten(2), x, mean, rstd, w, layout="map")
        return [out, one, *grads, dx, dw, db]

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        x.mul_(1.0 if turn == 0 else -0.7)
        want = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held)), turn


def test_tokens_refusals(device):
    x = torch.randn(2, 8, 16, device=device)
    with pytest.raises(TypeError):
        sconv.sconv_layernorm_forward(x.cpu())
    with pytest.raises(TypeError):
        sconv.sconv_layernorm_forward(x.half())
    with pytest.raises(TypeError):
        sconv.sconv_layernorm_forward(x.transpose(1, 2))
    with pytest.raises(ValueError):
        sconv.sconv_layernorm_forward(x, torch.ones(15, device=device))
    with pytest.raises(ValueError):
        sconv.sconv_layernorm_forward(x, layout="nchw")
    with pytest.raises(ValueError):
        sconv.sconv_layernorm_forward(x, out=torch.empty(2, 8, 15, device=device))
    with pytest.raises(sconv.SconvError):
        sconv.sconv_layernorm_forward(x, eps=-1.0)
    with pytest.raises(sconv.SconvError):
        sconv.sconv_layernorm_forward(x.to(BF16), out_dtype=F32)
    y, mean, rstd = sconv.sconv_layernorm_forward(x, stats=True)
    with pytest.raises(sconv.SconvError):
        sconv.sconv_layernorm_backward(y, x, mean, rstd, ws=torch.empty(16, dtype=torch.uint8, device=device))
    with pytest.raises(ValueError):
        sconv.sconv_layernorm_backward(y, x, mean[:1].contiguous(), rstd)
    q = torch.randn(2, 8, 2, 16, device=device)
    pos, freq = torch.zeros(8, 2, dtype=torch.int32, device=device), torch.ones(8, device=device)
    with pytest.raises(sconv.SconvError):
        sconv.sconv_rotary_forward(q, None, pos, freq, bytes([0] * 4 + [2] * 4))
    with pytest.raises(sconv.SconvError):
        sconv.sconv_rotary_forward(q, None, pos, torch.ones(9, device=device), bytes(9))
    with pytest.raises(ValueError):
        sconv.sconv_rotary_forward(q, None, pos, freq, bytes(7))
    with pytest.raises(TypeError):
        sconv.sconv_rotary_forward(q, None, pos.long(), freq, bytes(8))
    with pytest.raises(TypeError):
        sconv.sconv_rotary_forward(q, q.to(BF16), pos, freq, bytes(8))
    k, v, lam = torch.randn(2, 9, 2, 16, device=device), torch.randn(2, 9, 1, 32, device=device), torch.ones(1, device=device)
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan"))):
        with pytest.raises(sconv.SconvError):
            sconv.sconv_diffattn_forward(q, k, v, lam, **bad)
    with pytest.raises(ValueError):
        sconv.sconv_diffattn_forward(q, k, v[:, :8], lam)
    with pytest.raises(ValueError):
        sconv.sconv_diffattn_forward(q, k, v, torch.ones(2, device=device))
    with pytest.raises(TypeError):
        sconv.sconv_diffattn_forward(q, k, v, lam, k_lengths=torch.ones(2, device=device))
    with pytest.raises(ValueError):
        sconv.sconv_diffattn_forward(q, k, v, lam, k_mask=torch.ones(2, 8, dtype=torch.bool, device=device))
    with pytest.raises(sconv.SconvError):
        sconv.sconv_diffattn_forward(torch.randn(1, 2, 2, 136, device=device), torch.randn(1, 2, 2, 136, device=device),
                                     torch.randn(1, 2, 1, 16, device=device), lam)
    out, second, lse = sconv.sconv_diffattn_forward(q, k, v, lam, save=True)
    with pytest.raises(ValueError):
        sconv.sconv_diffattn_backward(out[:, :4].contiguous(), q, k, v, lam, out, second, lse)
    with pytest.raises(sconv.SconvError):
        sconv.sconv_diffattn_backward(out, q, k, v, lam, out, second, lse, ws=torch.empty(16, dtype=torch.uint8, device=device))
