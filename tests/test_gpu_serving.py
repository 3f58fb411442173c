"""The serving operators on the GPU against 64-bit references, at the sizes, types, strides and masks where they can go wrong."""
import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_1909_09927_amd as sconv  # noqa: E402
import serving_ref as ref  # noqa: E402
import tokens_ref  # noqa: E402
from serving_ref import E, E4M3, U, within  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [F32, BF16]
IDS = ["fp32", "bf16"]


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31) if all(isinstance(k, int) for k in key) else sum(map(ord, repr(key))))
    return g


def spread_rows(t, device, gap=3, lead=1):
    """The tensor [R, C] on the device with rows a gap apart, behind `lead` elements: at no aligned address."""
    R, C = t.shape
    buf = torch.full((lead + R * (C + gap),), float("nan") if t.is_floating_point() else 0, device=device).to(t.dtype)
    view = buf[lead:].view(R, C + gap)[:, :C]
    view.copy_(t)
    return view


# ---- 8-bit values

SHAPES8 = [(1, 1), (1, 128), (3, 127), (5, 130), (130, 8), (128, 128), (129, 1000), (257, 1031), (64, 4096)]


def awkward(M, K, dtype, g):
    """Values over many scales; blocks of zeros, of subnormals, of the largest; Inf and NaN; halves of steps."""
    x = torch.randn(M, K, generator=g) * torch.exp(3.0 * torch.randn(M, 1, generator=g))
    for m in range(0, M, 7):
        x[m] = 0.0
    for m in range(1, M, 11):
        x[m] *= 1e-38
    for m in range(2, M, 13):
        x[m] = torch.randint(-4000, 4000, (K,), generator=g) / 64.0
    x[-1, -1] = 448.0
    if M > 3:
        x[3, 0], x[3, -1], x[4 % M, K // 2], x[M // 2, 0] = float("inf"), float("nan"), -float("inf"), 3e38
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K", SHAPES8)
def test_quant8(device, M, K, rows, dtype):
    x = awkward(M, K, dtype, gen(M, K, rows))
    want, ws = ref.quant8(x, rows)
    for at in (x.to(device), spread_rows(x, device)):
        q, s = sconv.sconv_quant8(at, rows)
        assert q.dtype == E4M3 and s.shape == ws.shape
        assert np.array_equal(s.cpu().numpy(), ws)
        ref.same_bytes(q, want, "values")
    if rows == 1:
        q3, s3 = sconv.sconv_quant8(x.to(device).view(1, M, K))
        assert q3.shape == (1, M, K) and torch.equal(s3[0].cpu(), torch.from_numpy(ws))


def test_quant8_into_given_tensors_and_nothing(device):
    x = torch.randn(5, 200, generator=gen(1)).to(device)
    out = (torch.empty(5, 200, dtype=E4M3, device=device), torch.empty(5, 2, dtype=torch.uint8, device=device))
    got = sconv.sconv_quant8(x, out=out)
    assert got[0].data_ptr() == out[0].data_ptr() and got[1].data_ptr() == out[1].data_ptr()
    ref.same_bytes(out[0], ref.quant8(x.cpu())[0], "values")
    for shape in ((0, 5), (5, 0)):
        q, s = sconv.sconv_quant8(torch.empty(shape, device=device))
        assert q.shape == shape and s.shape == (shape[0], (shape[1] + 127) // 128)


# ---- root-mean-square norm

COMBOS = [(F32, None, F32), (F32, F32, F32), (F32, F32, BF16), (F32, F32, E4M3), (BF16, None, BF16), (BF16, BF16, BF16), (BF16, F32, BF16),
          (BF16, BF16, E4M3), (BF16, F32, E4M3), (BF16, None, E4M3), (F32, None, E4M3)]


@pytest.mark.parametrize("combo", COMBOS, ids=["-".join(str(t).replace("torch.", "") for t in c) for c in COMBOS])
@pytest.mark.parametrize("rows,C,spread", [(1, 1, False), (3, 100, True), (5, 128, False), (17, 129, True), (9, 512, False), (6, 1000, True), (1030, 2048, False), (4, 2056, True),
                                           (3, 8192, False), (2, 8200, False), (2, 16384, False), (5, 16383, True)])
def test_rmsnorm(device, rows, C, spread, combo):
    xt, rt, yt = combo
    g = gen(rows, C)
    x = (3.0 * torch.randn(rows, C, generator=g)).to(xt)
    res = None if rt is None else (torch.randn(rows, C, generator=g) - 0.5).to(rt)
    w = None if rows == 9 else (1.0 + 0.2 * torch.randn(C, generator=g)).to(xt if rows % 2 else F32)
    place = (lambda t: None if t is None else spread_rows(t, device)) if spread else (lambda t: None if t is None else t.to(device))
    xd, rd, wd = place(x), place(res), None if w is None else w.to(device)
    y, total, rstd = sconv.sconv_rmsnorm_forward(xd, wd, residual=rd, out_dtype=yt, stats=True, eps=1e-5)
    (wy, wt, wr), (by, bt, br) = ref.rmsnorm(x, res, w, float(np.float32(1e-5)), yt)
    within(rstd, wr, br, "rstd")
    assert (total is None) == (res is None)
    if res is not None:
        assert total.dtype == rt
        within(total, wt, bt, "total")
        mine = rd.clone() if not spread else place(res)
        y2, t2, r2 = sconv.sconv_rmsnorm_forward(xd, wd, residual=mine, out_dtype=yt, eps=1e-5, total=mine)
        assert t2.data_ptr() == mine.data_ptr() and torch.equal(t2, total) and r2 is None
        pairs = zip(y, y2) if yt == E4M3 else [(y, y2)]
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in pairs)
    if yt != E4M3:
        within(y, wy, by, "y")
        return
    q, s = y
    # a scale is that of a largest value within the bound of the wanted one
    tops, off = ref._block_tops(wy.numpy(), 1), ref._block_tops(by.numpy(), 1)
    got = s.cpu().numpy()
    assert got.shape == tops.shape and ((got >= ref.scale_byte(np.maximum(tops - off, 0))) & (got <= ref.scale_byte(tops + off))).all()
    step = 2.0 ** (s.cpu().double() - 127.0 - 10.0)[:, torch.arange(C) // 128]
    within(ref.held(q, s), wy, 1.01 * ref.HALF8 * wy.abs() + step + 2 * by, "y")


def test_rmsnorm_of_other_shapes(device):
    x = torch.randn(2, 3, 5, 64, generator=gen(2)).to(device)
    y, total, rstd = sconv.sconv_rmsnorm_forward(x, residual=x, stats=True)
    assert y.shape == total.shape == x.shape and rstd.shape == (2, 3, 5)
    one = sconv.sconv_rmsnorm_forward(x[0, 0, 0])[0]
    assert one.shape == (64,)
    none = sconv.sconv_rmsnorm_forward(x[:0], out_dtype=E4M3)[0]
    assert none[0].shape == (0, 3, 5, 64) and none[1].shape == (0, 3, 5, 1)
    with pytest.raises(TypeError):
        sconv.sconv_rmsnorm_forward(x.transpose(0, 1))
    with pytest.raises(ValueError):
        sconv.sconv_rmsnorm_forward(x, residual=x[:1])
    with pytest.raises(sconv.SconvError):
        sconv.sconv_rmsnorm_forward(x, out_dtype=torch.float16)
    with pytest.raises(sconv.SconvError):
        sconv.sconv_rmsnorm_forward(x.bfloat16(), out_dtype=F32)


def test_rmsnorm_rows_do_not_meet(device):
    """Inf and NaN stay in their rows, zeros of rows of zeros are zeros."""
    x = torch.randn(6, 300, generator=gen(3))
    x[1, 7], x[3, 299], x[4] = float("inf"), float("nan"), 0.0
    for dtype in (F32, E4M3):
        y = sconv.sconv_rmsnorm_forward(x.to(device), out_dtype=dtype)[0]
        y = ref.held(*y) if dtype == E4M3 else y.cpu().double()
        assert torch.isnan(y[3]).all() and torch.isnan(y[1, 7]) and (y[4] == 0).all() and torch.isfinite(y[[0, 2, 5]]).all()
        assert (y[1, :7] == 0).all()


GRADS = [(F32, F32, None), (F32, F32, F32), (BF16, F32, None), (BF16, F32, BF16), (BF16, BF16, None)]


@pytest.mark.parametrize("types", GRADS, ids=["dy-total-dx:" + "-".join(str(t).replace("torch.", "") for t in c) for c in GRADS])
@pytest.mark.parametrize("rows,C,spread,along", [(1, 1, False, False), (3, 100, True, True), (40, 128, False, True), (5000, 512, False, True), (33, 1000, True, False), (700, 2048, False, False),
                                                 (5, 4104, False, True), (3, 8200, True, True), (2, 16384, False, False)])
def test_rmsnorm_backward(device, rows, C, spread, along, types):
    gt, tt, xt = types
    g = gen(rows, C, 4)
    t = (2.0 * torch.randn(rows, C, generator=g)).to(tt)
    dy = torch.randn(rows, C, generator=g).to(gt)
    dt = torch.randn(rows, C, generator=g).to(tt) if along else None
    w = None if rows == 33 else (1.0 + 0.2 * torch.randn(C, generator=g)).to(BF16 if rows == 40 else F32)
    rstd = (1.0 / (t.double().square().mean(1) + 1e-5).sqrt()).float()
    place = (lambda v: None if v is None else spread_rows(v, device)) if spread else (lambda v: None if v is None else v.to(device))
    args = (place(dy), place(t), rstd.to(device), None if w is None else w.to(device), place(dt))
    dx, dres, dw = sconv.sconv_rmsnorm_backward(*args, x_dtype=xt)
    (d, wdw), (bd, bw) = ref.rmsnorm_grad(dy, t, rstd, w, dt)
    within(dres, d, bd + 1.01 * U[tt] * d.abs(), "dres")
    if xt in (None, tt):
        assert dx is dres
    else:
        assert dx.dtype == xt
        within(dx, d, bd + 1.01 * U[xt] * d.abs(), "dx")
    wtype = F32 if w is None else w.dtype
    assert dw.dtype == wtype
    within(dw, wdw, bw + 1.01 * U[wtype] * wdw.abs(), "dw")
    again = sconv.sconv_rmsnorm_backward(*args, x_dtype=xt)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dres, dw)))
    assert sconv.sconv_rmsnorm_backward(*args, x_dtype=xt, param_grads=False)[2] is None


def test_rmsnorm_backward_is_the_forwards(device):
    """Against differences of the forward call's formula in 64 bits, in random directions; the difference's own error is of the third order."""
    g = gen(5)
    x, res, w, dy = (torch.randn(7, 96, generator=g, dtype=torch.float64) for _ in range(4))
    w, eps = w[0], 1e-3
    x, res, w, dy = (t.float().double() for t in (x, res, w, dy))

    def loss(x, res, w):
        t = x + res
        return (t / (t.square().mean(1, keepdim=True) + eps).sqrt() * w * dy).sum()

    y, total, rstd = sconv.sconv_rmsnorm_forward(x.float().to(device), w.float().to(device), residual=res.float().to(device), eps=eps, stats=True)
    dx, dres, dw = (t.cpu().double() for t in sconv.sconv_rmsnorm_backward(dy.float().to(device), total, rstd, w.float().to(device)))
    h = 1e-4
    for k in range(3):
        a, b, c = (torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (x, res, w))
        diff = (loss(x + h * a, res + h * b, w + h * c) - loss(x - h * a, res - h * b, w - h * c)) / (2 * h)
        said = (dx * a).sum() + (dres * b).sum() + (dw * c).sum()
        # 1344 terms of order one in 32 bits: 60 roundings each
        assert abs(diff - said) <= 60 * E * ((dx * a).abs().sum() + (dres * b).abs().sum() + (dw * c).abs().sum()) + 1e-5, k


def test_rmsnorm_backward_of_no_rows(device):
    z = torch.zeros(0, 40, device=device)
    dx, dres, dw = sconv.sconv_rmsnorm_backward(z, z, z[:, 0].contiguous(), torch.ones(40, device=device))
    assert dx.shape == (0, 40) and (dw == 0).all()


# ---- the product

def operands(M, N, K, g):
    """8-bit operands whose scales differ from block to block, made on the host."""
    x = torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, (K + 127) // 128, generator=g))[:, torch.arange(K) // 128]
    w = torch.randn(N, K, generator=g) * torch.exp(torch.randn((N + 127) // 128, (K + 127) // 128, generator=g))[torch.arange(N) // 128][:, torch.arange(K) // 128]
    out = []
    for t, rows in ((x, 1), (w, 128)):
        q, s = ref.quant8(t, rows)
        out.append((torch.from_numpy(q).view(E4M3), torch.from_numpy(s)))
    return out


LINEAR = [(1, 1, 1), (1, 16, 128), (2, 17, 129), (16, 1000, 256), (17, 64, 1024), (33, 130, 383), (64, 2048, 2048), (5, 4200, 300), (30, 4100, 200), (50, 5000, 130), (65, 128, 128), (65, 1, 1), (100, 129, 200), (128, 256, 512),
          (200, 1000, 896), (257, 300, 1040), (300, 136, 4096), (1000, 520, 640), (784, 1024, 384), (4100, 4099, 400), (4096, 4096, 256),
          (2304, 9000, 144), (5000, 4300, 64), (9000, 9000, 80), (70, 130, 15500), (66, 40, 31000)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear8(device, M, N, K, dtype):
    (xq, xs), (wq, ws) = operands(M, N, K, gen(M, N, K))
    want, bound = ref.linear8(ref.held(xq, xs), ref.held(wq, ws, 128), dtype, (xs, ws) if dtype == BF16 and M > 16 else None)
    x, w = (xq.to(device), xs.to(device)), (wq.to(device), ws.to(device))
    y = sconv.sconv_linear8(x, w, out_dtype=dtype)
    assert y.dtype == dtype
    within(y, want, bound, "y")
    # what is cut off has the products' random signs: of the whole it is far less than the bound of each (2^-13 of the largest of eight, a product)
    if M * N > 1000:
        assert (y.cpu().double() - want).norm() <= (U[dtype] + (2.0 ** -11 if dtype == BF16 else (K + 16) * E)) * want.norm()
    assert torch.equal(y, sconv.sconv_linear8(x, w, out_dtype=dtype))
    # rows at no aligned address; the result is the same but for what another kernel's order of sums does
    odd = [(spread_rows(q.view(torch.uint8), device).view(E4M3), s.to(device)) for q, s in ((xq, xs), (wq, ws))]
    within(sconv.sconv_linear8(*odd, out_dtype=dtype), want, bound, "y of odd rows")
    # rows a whole vector apart, in part of a larger tensor
    big = [(torch.zeros(q.shape[0], (K + 31) // 16 * 16, dtype=torch.uint8, device=device), q, s) for q, s in ((xq, xs), (wq, ws))]
    wide = []
    for buf, q, s in big:
        buf.fill_(127)                                     # (NaN beside the rows)
        buf[:, :K] = q.to(device).view(torch.uint8)
        wide.append((buf[:, :K].view(E4M3), s.to(device)))
    within(sconv.sconv_linear8(*wide, out_dtype=dtype), want, bound, "y of rows with NaN behind them")


def test_linear8_shapes_and_corners(device):
    (xq, xs), (wq, ws) = operands(12, 40, 256, gen(6))
    x, w = (xq.to(device), xs.to(device)), (wq.to(device), ws.to(device))
    y = sconv.sconv_linear8(x, w)
    y3 = sconv.sconv_linear8((x[0].view(3, 4, 256), x[1].view(3, 4, 2)), w)
    assert torch.equal(y3.view(12, 40), y)
    out = torch.empty(12, 40, dtype=BF16, device=device)
    assert sconv.sconv_linear8(x, w, out=out).data_ptr() == out.data_ptr() and torch.equal(out, y)
    empty = (torch.empty(12, 0, dtype=E4M3, device=device), torch.empty(12, 0, dtype=torch.uint8, device=device))
    none = (torch.empty(40, 0, dtype=E4M3, device=device), torch.empty(1, 0, dtype=torch.uint8, device=device))
    assert (sconv.sconv_linear8(empty, none) == 0).all()
    assert sconv.sconv_linear8((x[0][:0], x[1][:0]), w).shape == (0, 40)
    with pytest.raises(ValueError):
        sconv.sconv_linear8(x, (w[0], w[1][:, :1].contiguous()))
    with pytest.raises(TypeError):
        sconv.sconv_linear8((x[0].float(), x[1]), w)


@pytest.mark.parametrize("M", [5, 100])
def test_linear8_nan_stays_in_its_row_and_column(device, M):
    (xq, xs), (wq, ws) = operands(M, 150, 300, gen(7, M))
    xq.view(torch.uint8)[3, 290], wq.view(torch.uint8)[149, 0] = 0x7f, 0xff
    y = sconv.sconv_linear8((xq.to(device), xs.to(device)), (wq.to(device), ws.to(device))).cpu()
    nan = torch.zeros(M, 150, dtype=torch.bool)
    nan[3], nan[:, 149] = True, True
    assert torch.equal(torch.isnan(y), nan)


@pytest.mark.parametrize("M", [5, 100])
def test_linear8_of_far_scales(device, M):
    """Blocks of the smallest and largest scales that are made, whose product has an ordinary size."""
    (xq, xs), (wq, ws) = operands(M, 20, 256, gen(8, M))
    xs[:, 0], ws[:, 0], xs[:, 1], ws[:, 1] = 1, 247, 240, 10
    want, bound = ref.linear8(ref.held(xq, xs), ref.held(wq, ws, 128), F32)
    within(sconv.sconv_linear8((xq.to(device), xs.to(device)), (wq.to(device), ws.to(device)), out_dtype=F32), want, bound, "y")


# ---- the cache

def new_cache(device, g, B, per, page, Hk, D, Hv, Dv, dtype, heads_first=True, spare=2, fill=None, width=None):
    """A cache whose requests have per[b] pages, in no order, among others that are nobody's; table entries behind them are -1 or wild."""
    total = sum(per) + spare
    width = max(per) + 1 if width is None else width
    order = torch.randperm(total, generator=g).int()
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[:, ::2] = total + 5
    at = 0
    for b in range(B):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]

    def pages(H, *last, kind):
        t = torch.randint(0, 256, (total, page, H, *last), generator=g, dtype=torch.uint8) if kind != "scale" else torch.randint(100, 150, (total, page, H), generator=g, dtype=torch.uint8)
        if kind == E4M3:
            t = t.view(E4M3)
        elif kind != "scale":
            t = torch.full((total, page, H, *last), float("nan"), dtype=kind) if fill is None else torch.full((total, page, H, *last), fill, dtype=kind)
        if heads_first:
            t = t.view(torch.uint8).transpose(1, 2).contiguous().to(device).view(E4M3).transpose(1, 2) if kind == E4M3 else t.transpose(1, 2).contiguous().to(device).transpose(1, 2)
            return t
        return t.to(device)

    quantised = dtype == E4M3
    return sconv.PagedCache(pages(Hk, D, kind=dtype), pages(Hv, Dv, kind=dtype), table.to(device), pages(Hk, kind="scale") if quantised else None,
                            pages(Hv, kind="scale") if quantised else None)


def raw(t):
    return None if t is None else t.cpu().contiguous().view(torch.uint8).clone()


CACHES = [(1, 1, 1, 1, 8, 1, 8), (3, 1, 16, 4, 64, 2, 128), (2, 37, 20, 2, 30, 1, 61), (4, 5, 7, 8, 128, 4, 256), (2, 130, 64, 6, 16, 3, 200), (5, 3, 100, 2, 1, 1, 3)]


@pytest.mark.parametrize("heads_first", [True, False])
@pytest.mark.parametrize("dtype,kept", [(F32, E4M3), (BF16, E4M3), (F32, F32), (BF16, BF16)], ids=["fp32-e4m3", "bf16-e4m3", "fp32", "bf16"])
@pytest.mark.parametrize("B,S,page,Hk,D,Hv,Dv", CACHES)
def test_cache_write_and_read(device, B, S, page, Hk, D, Hv, Dv, dtype, kept, heads_first):
    g = gen(B, S, page)
    starts = torch.randint(0, 3 * page, (B,), generator=g)
    counts = torch.randint(0, S + 1, (B,), generator=g)
    counts[0] = S
    if B > 2:
        starts[2] = -2                                     # (its first two tokens have no position)
    per = [max(1, int(s + n + page - 1) // page) for s, n in zip(starts, counts)]
    if B > 1:
        per[1] = max(1, per[1] - 1)                        # (its last page is missing)
    cache = new_cache(device, g, B, per, page, Hk, D, Hv, Dv, kept, heads_first)
    # slices of one projection's output
    row = torch.randn(B, S, Hk * D + Hv * Dv + 5, generator=g).to(dtype)
    dev = row.to(device)
    k, v = dev[:, :, :Hk * D].unflatten(2, (Hk, D)), dev[:, :, Hk * D:Hk * D + Hv * Dv].unflatten(2, (Hv, Dv))
    want = [raw(t) for t in cache]
    table = cache.table.cpu()
    pages = cache.k.shape[0]
    held = [torch.zeros(B, S, Hk, D, dtype=torch.float64), torch.zeros(B, S, Hv, Dv, dtype=torch.float64)]
    for i, x in enumerate((k.cpu(), v.cpu())):
        H, W = x.shape[2:]
        for b in range(B):
            for s in range(int(counts[b])):
                at = int(starts[b]) + s
                if at < 0 or at >= table.shape[1] * page or not 0 <= int(table[b, at // page]) < pages:
                    continue
                p = int(table[b, at // page])
                if kept == E4M3:
                    q, e = ref.quant8(torch.nn.functional.pad(x[b, s], (0, 0)) if W <= 128 else x[b, s].reshape(H, W)[:, :W], 1)
                    if W > 128:                            # (one scale for the whole head)
                        e = ref.scale_byte(np.abs(x[b, s].double().numpy()).max(1))[:, None]
                        q = ref._to8(x[b, s].double().numpy() * 2.0 ** (127.0 - e))
                    want[i][p, at % page] = torch.from_numpy(q)
                    want[3 + i][p, at % page] = torch.from_numpy(e[:, 0].astype(np.uint8))
                    held[i][b, s] = torch.from_numpy(ref.VALUES8[q] * 2.0 ** (e.astype(np.float64) - 127.0))
                else:
                    want[i].view(pages, page, H, -1)[p, at % page] = x[b, s].contiguous().view(torch.uint8).view(H, -1)
                    held[i][b, s] = x[b, s].double()
    si, ci = starts.int().to(device), counts.int().to(device)
    sconv.sconv_cache_write(cache, k, v, si, ci)
    for name, got, w in zip(cache._fields, cache, want):
        if w is not None:
            assert torch.equal(raw(got), w), f"{name}: not the bytes that were wanted"
    for out in ([dtype] if kept != E4M3 else [BF16, F32]):
        rk, rv = sconv.sconv_cache_read(cache, S, si, ci, out_dtype=out)
        assert rk.dtype == out and torch.equal(rk.cpu().double(), held[0]) and torch.equal(rv.cpu().double(), held[1])


def test_cache_calls_of_nothing(device):
    cache = sconv.sconv_cache_new(2, 0, 0, 16, 2, 8, 1, 8, device=device)
    one = torch.zeros(2, dtype=torch.int32, device=device)
    k, v = torch.ones(2, 3, 2, 8, device=device), torch.ones(2, 3, 1, 8, device=device)
    sconv.sconv_cache_write(cache, k, v, one)
    rk, rv = sconv.sconv_cache_read(cache, 3, one)
    assert (rk == 0).all() and (rv == 0).all() and rk.shape == k.shape
    rk, rv = sconv.sconv_cache_read(cache, 0, one)
    assert rk.shape == (2, 0, 2, 8)
    q = torch.ones(2, 1, 2, 8, device=device)
    assert (sconv.sconv_diffattn_paged(q, cache, torch.ones(1, device=device), one + 5) == 0).all()
    assert sconv.sconv_diffattn_paged(q[:, :0], cache, torch.ones(1, device=device), one).shape == (2, 0, 1, 8)


def test_cache_refuses_what_does_not_fit(device):
    cache = sconv.sconv_cache_new(2, 4, 8, 16, 2, 8, 1, 8, device=device)
    starts = torch.zeros(2, dtype=torch.int32, device=device)
    k, v = torch.ones(2, 3, 2, 8, device=device), torch.ones(2, 3, 1, 8, device=device)
    for bad in (lambda: sconv.sconv_cache_write(cache, k[:1], v[:1], starts[:1]), lambda: sconv.sconv_cache_write(cache, k, v, starts.long()),
                lambda: sconv.sconv_cache_write(cache, k, v.bfloat16(), starts), lambda: sconv.sconv_cache_write(cache, k[:, :, :1], v, starts),
                lambda: sconv.sconv_cache_write(cache, k, v, starts, starts[:1]), lambda: sconv.sconv_cache_write(cache._replace(k_scales=None), k, v, starts),
                lambda: sconv.sconv_cache_write(cache._replace(table=cache.table.long()), k, v, starts),
                lambda: sconv.sconv_cache_write(cache._replace(k=cache.k.float(), v=cache.v.float()), k, v, starts),
                lambda: sconv.sconv_cache_write(cache._replace(v=cache.v[:4]), k, v, starts),
                lambda: sconv.sconv_diffattn_paged(k, cache, torch.ones(2, device=device), starts),
                lambda: sconv.sconv_diffattn_paged(k[:, :, :1], cache, torch.ones(1, device=device), starts)):
        with pytest.raises((TypeError, ValueError)):
            bad()


# ---- attention over it

def attend(q, cache, lam, lengths, scale, causal):
    """The reference over gathered keys, request by request: results and bounds."""
    B, Sq = q.shape[:2]
    outs, errs = [], []
    for b in range(B):
        k, v, ok = ref.gathered(cache, lengths, b)
        n = k.shape[0]
        as32 = [t.float().unsqueeze(0) for t in (k, v)]
        r, e = tokens_ref.attention(q[b:b + 1].cpu(), *as32, lam.cpu(), scale, causal, None, ok.unsqueeze(0))
        outs.append(r["out"])
        errs.append(e["out"])
    return torch.cat(outs), torch.cat(errs)


def filled(device, g, lengths, page, Hkv, D, Dv, dtype, kept, heads_first, width=None):
    """A cache with keys and values in every position, NaN or anything in all other slots."""
    B = len(lengths)
    per = [max(0, -(-n // page)) for n in lengths]
    cache = new_cache(device, g, B, per, page, 2 * Hkv, D, Hkv, Dv, kept, heads_first, width=width)
    S = max(max(lengths), 1)
    k, v = torch.randn(B, S, 2 * Hkv, D, generator=g).to(dtype).to(device), torch.randn(B, S, Hkv, Dv, generator=g).to(dtype).to(device)
    sconv.sconv_cache_write(cache, k, v, torch.zeros(B, dtype=torch.int32, device=device), torch.tensor(lengths, dtype=torch.int32, device=device))
    return cache


#       lengths, Sq, H, Hkv, D, Dv, page, causal
ATTN = [([1], 1, 1, 1, 8, 8, 1, False), ([0, 1, 33], 1, 2, 1, 64, 128, 16, True), ([5, 700, 0, 64], 1, 8, 2, 64, 128, 16, True), ([100, 31], 5, 4, 2, 32, 64, 20, True),
        ([300, 299, 17, 1], 3, 4, 4, 74, 148, 24, True), ([1000], 1, 16, 1, 128, 256, 64, False), ([257, 512], 9, 8, 2, 64, 128, 32, True), ([90, 2], 4, 24, 3, 40, 33, 7, True),
        ([400, 45], 2, 64, 2, 32, 64, 16, True), ([2500, 3, 1900], 1, 4, 2, 16, 32, 100, False), ([130, 64], 3, 20, 1, 128, 128, 48, True), ([70, 70], 6, 3, 3, 9, 13, 5, True),
        ([513, 40], 1, 2, 2, 96, 192, 16, False), ([6000], 2, 2, 1, 64, 64, 256, True)]


@pytest.mark.parametrize("dtype,kept", [(F32, E4M3), (BF16, E4M3), (F32, F32), (BF16, BF16)], ids=["fp32-e4m3", "bf16-e4m3", "fp32", "bf16"])
@pytest.mark.parametrize("case", ATTN, ids=lambda c: "-".join(map(str, c[1:])) + "-n" + "_".join(map(str, c[0])))
def test_paged(device, case, dtype, kept):
    lengths, Sq, H, Hkv, D, Dv, page, causal = case
    g = gen(*map(int, case[1:7]))
    cache = filled(device, g, lengths, page, Hkv, D, Dv, dtype, kept, heads_first=(Sq + H) % 2 == 0)
    B = len(lengths)
    # queries as slices of a projection's output
    q = (1.5 * torch.randn(B, Sq, 2 * H * D + 7, generator=g)).to(dtype).to(device)[:, :, 3:3 + 2 * H * D].unflatten(2, (2 * H, D))
    lam = 0.3 + 0.2 * torch.randn(H, generator=g).to(device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    want, bound = attend(q, cache, lam, lengths, None, causal)
    got = sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal)
    within(got, want, bound, "out")
    assert torch.equal(got, sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal))
    ws = torch.empty(0, dtype=torch.uint8, device=device)
    within(sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal, ws=ws), want, bound, "out, a workgroup a request")
    out = torch.empty_like(got)
    need = sconv.sconv_diffattn_paged_workspace_size(q, cache, lam, n)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=device)     # (NaN in every part)
    assert torch.equal(sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal, out=out, ws=ws), got) and out.data_ptr() != got.data_ptr()


@pytest.mark.parametrize("kept", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 12])
def test_paged_pages_that_are_not_there(device, page, kept):
    """Missing pages in the middle, at the ends and everywhere; lengths below 0 and past the table."""
    g = gen(9, page)
    lengths = [200, 200, 150, 100, 90]
    cache = filled(device, g, lengths, page, 2, 64, 128, BF16, kept, True)
    table = cache.table.clone()
    table[0, 3], table[0, 0], table[1, :] = -1, 1 << 30, -7
    table[2, 1::2] = cache.k.shape[0]
    cache = cache._replace(table=table)
    said = [200, 200, 150, -3, 1 << 30]
    q, lam = torch.randn(5, 2, 8, 64, generator=g).to(BF16).to(device), torch.full((4,), 0.5, device=device)
    got = sconv.sconv_diffattn_paged(q, cache, lam, torch.tensor(said, dtype=torch.int32, device=device), causal=True)
    want, bound = attend(q, cache, lam, said, None, True)
    assert (want[1] == 0).all() and (want[3] == 0).all() and torch.isfinite(want[:4]).all()
    within(got[:4], want[:4], bound[:4], "out")
    # the last request's length takes in slots of its last page that nobody wrote: NaN as the formulas have it
    nan = torch.isnan(want[4])
    assert torch.equal(torch.isnan(got[4].cpu()), nan)
    within(torch.where(nan, 0.0, got[4].cpu().double()), torch.where(nan, 0.0, want[4]), torch.where(nan, 0.0, bound[4]), "out of slots nobody wrote")


def test_paged_many_requests_and_spare_capacity(device):
    """Lengths from none to long under a table far wider than any of them."""
    g = gen(10)
    lengths = [int(n) for n in torch.randint(0, 90, (150,), generator=g)]
    lengths[7], lengths[70], lengths[149] = 3000, 0, 1
    cache = filled(device, g, lengths, 16, 1, 32, 64, BF16, E4M3, True, width=5000)
    q, lam = torch.randn(150, 1, 4, 32, generator=g).to(BF16).to(device), torch.full((2,), 0.4, device=device)
    got = sconv.sconv_diffattn_paged(q, cache, lam, torch.tensor(lengths, dtype=torch.int32, device=device), causal=True)
    want, bound = attend(q, cache, lam, lengths, None, True)
    within(got, want, bound, "out")


@pytest.mark.parametrize("page", [16, 20])
def test_paged_many_short_requests(device, page):
    """So many that no request is split: the same answers with scratch and without."""
    g = gen(16, page)
    lengths = [int(n) for n in torch.randint(0, 120, (300,), generator=g)]
    lengths[5], lengths[6] = 400, 0
    cache = filled(device, g, lengths, page, 8, 32, 64, BF16, E4M3, True)
    q, lam = torch.randn(300, 1, 16, 32, generator=g).to(BF16).to(device), torch.full((8,), 0.4, device=device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    got = sconv.sconv_diffattn_paged(q, cache, lam, n, causal=True)
    want, bound = attend(q, cache, lam, lengths, None, True)
    within(got, want, bound, "out")
    assert sconv.sconv_diffattn_paged_workspace_size(q, cache, lam, n) == 0
    # a wider table of the same positions: split
    wide = torch.full((300, 2000), -1, dtype=torch.int32, device=device)
    wide[:, :cache.table.shape[1]] = cache.table
    split = cache._replace(table=wide)
    assert sconv.sconv_diffattn_paged_workspace_size(q, split, lam, n) > 0
    within(sconv.sconv_diffattn_paged(q, split, lam, n, causal=True), want, bound, "out, split")


def test_paged_scale_and_large_scores(device):
    g = gen(11)
    cache = filled(device, g, [300, 77], 16, 2, 64, 128, F32, F32, False)
    q, lam = (30.0 * torch.randn(2, 1, 8, 64, generator=g)).to(device), torch.full((4,), 0.7, device=device)
    n = torch.tensor([300, 77], dtype=torch.int32, device=device)
    for scale in (0.02, 1.0):
        got = sconv.sconv_diffattn_paged(q, cache, lam, n, scale=scale)
        want, bound = attend(q, cache, lam, [300, 77], scale, False)
        within(got, want, bound, "out")


#       lengths, Sq, H, Hkv, D, Dv, page: up to eight rows of a key head, pages of whole 16 slots
FEW = [([700, 16, 0, 17], 1, 2, 2, 128, 256, 16), ([130, 1000], 2, 8, 2, 128, 128, 32), ([333, 64, 1], 1, 8, 1, 32, 64, 48), ([40] * 70, 1, 4, 4, 64, 128, 16), ([2000, 5], 8, 1, 1, 64, 256, 64)]


@pytest.mark.parametrize("heads_first", [True, False], ids=["heads-first", "slots-first"])
@pytest.mark.parametrize("dtype,kept", [(F32, E4M3), (BF16, E4M3), (F32, F32), (BF16, BF16)], ids=["fp32-e4m3", "bf16-e4m3", "fp32", "bf16"])
@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c[1:])) + "-n" + "_".join(map(str, c[0][:4])))
def test_paged_few_rows(device, case, dtype, kept, heads_first):
    lengths, Sq, H, Hkv, D, Dv, page = case
    g = gen(*case[1:])
    cache = filled(device, g, lengths, page, Hkv, D, Dv, dtype, kept, heads_first=heads_first)
    q = torch.randn(len(lengths), Sq, 2 * H, D, generator=g).to(dtype).to(device)
    lam = 0.3 + 0.2 * torch.randn(H, generator=g).to(device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    for causal in (True, False):
        want, bound = attend(q, cache, lam, lengths, None, causal)
        within(sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal), want, bound, f"out, causal {causal}")


@pytest.mark.parametrize("kept", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("off", [1, 4, 8])
def test_paged_pages_at_odd_addresses(device, off, kept):
    """Pools and scales that begin inside an allocation: the same results from any address."""
    g = gen(13, off)
    cache = filled(device, g, [300, 33], 16, 2, 64, 128, BF16, kept, True)
    q, lam = torch.randn(2, 1, 8, 64, generator=g).to(BF16).to(device), torch.full((4,), 0.5, device=device)
    n = torch.tensor([300, 33], dtype=torch.int32, device=device)

    def moved(t, by):
        if t is None:
            return None
        buf = torch.empty(t.numel() + 32, dtype=t.dtype, device=device)
        to = buf[by:by + t.numel()].as_strided(t.shape, t.stride())
        to.copy_(t)
        return to

    want, bound = attend(q, cache, lam, [300, 33], None, True)
    for which in ("k", "v", "k_scales", "v_scales"):
        got = sconv.sconv_diffattn_paged(q, cache._replace(**{which: moved(getattr(cache, which), off)}), lam, n, causal=True)
        within(got, want, bound, which)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("page", [16, 12])
def test_paged_of_far_scales(device, page, dtype):
    """Values near both ends of 32 bits, and both in one request.  Scores near 0: weights near 1, whose sum of products stays in range."""
    g = gen(14, page)
    lengths = [100, 70, 90]
    cache = filled(device, g, lengths, page, 2, 64, 128, dtype, E4M3, True)
    v, vs = cache.v, cache.v_scales.clone()
    small = torch.randint(1, 3, v.shape, generator=g) + 128 * torch.randint(0, 2, v.shape, generator=g)           # 2^-9, 2^-8, either sign
    large = torch.randint(0x70, 0x7f, v.shape, generator=g) + 128 * torch.randint(0, 2, v.shape, generator=g)     # 128 .. 448
    own = torch.full_like(v.view(torch.uint8), 127)
    table = cache.table.cpu()
    for b, (bytes_, scale) in enumerate(((small, 254), (large, 1), (small, 0))):
        for p in table[b][:-(-lengths[b] // page)].tolist():
            own[p] = bytes_[p].to(torch.uint8).to(device)
            vs[p] = scale or torch.tensor([254, 1], dtype=torch.uint8).repeat(page)[:page, None].to(device)
    cache = cache._replace(v=own.view(E4M3), v_scales=vs)
    q, lam = (0.01 * torch.randn(3, 1, 8, 64, generator=g)).to(dtype).to(device), torch.full((4,), 0.5, device=device)
    want, bound = attend(q, cache, lam, lengths, None, True)
    # an addition of the matrix pipe may take what is below the smallest normal number, 2^-126, as 0: three pieces, a term a key
    bound = bound + 3 * 100 * 1.5 * 2.0 ** -126
    within(sconv.sconv_diffattn_paged(q, cache, lam, torch.tensor(lengths, dtype=torch.int32, device=device), causal=True), want, bound, "out")


@pytest.mark.parametrize("kept", [BF16, E4M3], ids=["bf16", "e4m3"])
def test_paged_offsets_past_32_bits(device, kept):
    """A pool of more than 2^32 elements whose last pages are used, by every call on a cache."""
    page, Hkv, D, Dv, total = 64, 4, 64, 128, 140000
    g = gen(12)
    k = torch.empty(total, 2 * Hkv, page, D, dtype=kept, device=device).transpose(1, 2)
    v = torch.empty(total, Hkv, page, Dv, dtype=kept, device=device).transpose(1, 2)
    assert k.numel() > 1 << 32
    ks = torch.empty(total, 2 * Hkv, page, dtype=torch.uint8, device=device).transpose(1, 2) if kept == E4M3 else None
    vs = torch.empty(total, Hkv, page, dtype=torch.uint8, device=device).transpose(1, 2) if kept == E4M3 else None
    table = torch.tensor([[total - 1, 0, total - 3, total // 2 + 7]], dtype=torch.int32, device=device)
    cache = sconv.PagedCache(k, v, table, ks, vs)
    nk, nv = torch.randn(1, 250, 2 * Hkv, D, generator=g).to(BF16).to(device), torch.randn(1, 250, Hkv, Dv, generator=g).to(BF16).to(device)
    zero = torch.zeros(1, dtype=torch.int32, device=device)
    sconv.sconv_cache_write(cache, nk, nv, zero)
    rk, rv = sconv.sconv_cache_read(cache, 250, zero)
    small = sconv.sconv_cache_new(1, 4, 4, page, 2 * Hkv, D, Hkv, Dv, dtype=kept, device=device)
    small.table.copy_(torch.arange(4, dtype=torch.int32)[None])
    sconv.sconv_cache_write(small, nk, nv, zero)
    sk, sv = sconv.sconv_cache_read(small, 250, zero)
    assert torch.equal(rk, sk) and torch.equal(rv, sv)
    q, lam, n = torch.randn(1, 1, 8, D, generator=g).to(BF16).to(device), torch.full((4,), 0.5, device=device), zero + 250
    assert torch.equal(sconv.sconv_diffattn_paged(q, cache, lam, n), sconv.sconv_diffattn_paged(q, small, lam, n))
    del k, v, ks, vs, cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("H", [4, 24])
@pytest.mark.parametrize("page", [16, 12])
def test_paged_infinities_and_nan_stay_where_they_are(device, page, H):
    """A query of NaN makes its own row NaN and no other; a key of -Inf in one map loses its weight in that map alone."""
    g = gen(15, page, H)
    lengths = [200, 40]
    cache = filled(device, g, lengths, page, 2, 64, 128, BF16, BF16, True)
    q, lam = torch.randn(2, 1, 2 * H, 64, generator=g).abs().to(BF16).to(device), torch.full((H,), 0.5, device=device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    want, bound = attend(q, cache, lam, lengths, None, True)
    bad = q.clone()
    bad[0, 0, 2 * 1 + 1, 5] = float("nan")
    got = sconv.sconv_diffattn_paged(bad, cache, lam, n, causal=True).cpu()
    assert torch.isnan(got[0, 0, 1]).all()
    keep = torch.ones(2, 1, H, dtype=torch.bool)
    keep[0, 0, 1] = False
    within(got[keep], want[keep], bound[keep], "rows beside a NaN")
    # position 37 of request 0: the first map's key of key head 1 (queries are positive, so its scores are -Inf)
    at = int(cache.table[0, 37 // page])
    cache.k[at, 37 % page, 2, 7] = -float("inf")
    got = sconv.sconv_diffattn_paged(q, cache, lam, n, causal=True).cpu().double()
    within(got[1], want[1], bound[1], "the other request")
    k, v, _ = ref.gathered(cache, lengths, 0)
    G, qd = H // 2, q[0, 0].cpu().double()
    for h in range(H):
        w = [torch.softmax((k[:, 2 * (h // G) + m] @ qd[2 * h + m]) / 8.0, 0) for m in (0, 1)]
        exact = (w[0] - 0.5 * w[1]) @ v[:, h // G]
        # the result's rounding, and 2^-16 of every weight (two 16-bit values; scores and sums in 32 bits are far closer)
        err = exact.abs() * U[BF16] + (w[0] + 0.5 * w[1]) @ v[:, h // G].abs() * 2.0 ** -14
        assert torch.isfinite(exact).all() and ((got[0, 0, h] - exact).abs() <= err).all(), h


def test_paged_the_longest_length(device):
    """2^31 - 1 positions in one page: equal scores, so a head's answer is the mean of its values, sums of 2^31 - 1 terms."""
    n = (1 << 31) - 1
    k, v = torch.zeros(1, n, 2, 1, dtype=BF16, device=device), torch.ones(1, n, 1, 1, dtype=BF16, device=device)
    table = torch.zeros(1, 1, dtype=torch.int32, device=device)
    cache = sconv.PagedCache(k, v, table)
    q, lam = torch.ones(1, 2, 2, 1, dtype=BF16, device=device), torch.tensor([0.25], device=device)
    length = torch.tensor([n], dtype=torch.int32, device=device)
    got = sconv.sconv_diffattn_paged(q, cache, lam, length, causal=True)
    # (1 - 0.25, which 16 bits hold; sums of ones are whole numbers below 2^24 a lane, their quotients and join within 2^-20)
    assert got.shape == (1, 2, 1, 1) and ((got.double() - 0.75).abs() <= 0.75 * U[BF16]).all()
    # the last position, seen by the last query alone
    v[0, -1] = float("inf")
    got = sconv.sconv_diffattn_paged(q[:, 1:], cache, lam, length, causal=True)
    assert not torch.isfinite(got).any()
    got = sconv.sconv_diffattn_paged(q[:, 1:], cache, lam, length - 1, causal=True)
    assert ((got.double() - 0.75).abs() <= 0.75 * U[BF16]).all()
    rk, rv = sconv.sconv_cache_read(cache, 3, length - 3)
    assert torch.isinf(rv[0, 2]).all() and (rv[0, :2] == 1).all() and (rk == 0).all()
    del k, v, cache
    torch.cuda.empty_cache()


# ---- together

def step(x, res, w, w_in, w_out, cache, lens, lam, freq, axes, H, Hkv, D, Dv):
    """One token of every request: norm, projection, positions, cache, attention, projection."""
    h, total, _ = sconv.sconv_rmsnorm_forward(x, w, residual=res, out_dtype=E4M3)
    row = sconv.sconv_linear8(h, w_in).unsqueeze(1)
    a, b = 2 * H * D, 2 * (H + Hkv) * D
    q, k, v = row[..., :a].unflatten(-1, (2 * H, D)), row[..., a:b].unflatten(-1, (2 * Hkv, D)), row[..., b:].unflatten(-1, (Hkv, Dv))
    q, k = sconv.sconv_rotary_forward(q, k, lens.view(-1, 1, 1), freq, axes)
    sconv.sconv_cache_write(cache, k, v, lens)
    o = sconv.sconv_diffattn_paged(q, cache, lam, lens + 1, causal=True)
    o = sconv.sconv_rmsnorm_forward(o, out_dtype=BF16)[0]
    return sconv.sconv_linear8(sconv.sconv_quant8(o.view(x.shape[0], H * Dv)), w_out), total, q


def step_state(device, seed, B=6, C=256, H=4, Hkv=2, D=32, Dv=64, page=16):
    g = gen(13, seed)
    lens = torch.randint(0, 60, (B,), generator=g).int()
    per = [int(n) // page + 1 for n in lens]
    cache = new_cache(device, g, B, per, page, 2 * Hkv, D, Hkv, Dv, E4M3)
    w_in = sconv.sconv_quant8((torch.randn(2 * (H + Hkv) * D + Hkv * Dv, C, generator=g) / 16).to(device), 128)
    w_out = sconv.sconv_quant8((torch.randn(C, H * Dv, generator=g) / 16).to(device), 128)
    k, v = torch.randn(B, 60, 2 * Hkv, D, generator=g).to(BF16).to(device), torch.randn(B, 60, Hkv, Dv, generator=g).to(BF16).to(device)
    lens = lens.to(device)
    sconv.sconv_cache_write(cache, k, v, torch.zeros_like(lens), lens)
    return dict(x=torch.randn(B, C, generator=g).to(BF16).to(device), res=torch.randn(B, C, generator=g).to(device), w=torch.ones(C, device=device), w_in=w_in, w_out=w_out,
                cache=cache, lens=lens, lam=torch.full((H,), 0.4, device=device), freq=torch.tensor([50.0 ** (-i / 16) for i in range(16)], device=device),
                axes=sconv.sconv_rotary_axes((16,)), H=H, Hkv=Hkv, D=D, Dv=Dv)


def test_a_step_against_its_definition(device):
    """Each call's result against the 64-bit reference over what the calls before it gave."""
    s = step_state(device, 0)
    y, total, q = step(**s)
    lens = (s["lens"] + 1).tolist()
    want, bound = attend(q, s["cache"], s["lam"], lens, None, True)
    o = sconv.sconv_diffattn_paged(q, s["cache"], s["lam"], s["lens"] + 1, causal=True)
    within(o, want, bound, "attention")
    (wt, bt) = (s["x"].cpu().double() + s["res"].cpu().double(),) * 2
    within(total, wt, 2 * E * bt.abs(), "total")
    n = sconv.sconv_rmsnorm_forward(o, out_dtype=BF16)[0].view(6, -1).cpu()
    qn, sn = ref.quant8(n)
    wy, by = ref.linear8(ref.held(torch.from_numpy(qn), torch.from_numpy(sn)), ref.held(*s["w_out"], 128), BF16)
    within(y, wy, by, "y")


def test_a_step_captured_and_replayed(device):
    """The step in a graph, replayed with other inputs, eager work and synchronisations between; two graphs keep scratch of their own."""
    states = [step_state(device, i) for i in (1, 2)]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in states:
            step(**s)
    torch.cuda.current_stream().wait_stream(side)
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(**s))
        graphs.append(graph)
    for turn in range(3):
        for s, graph, out in zip(states, graphs, outs):
            s["x"].copy_(torch.randn(s["x"].shape, generator=gen(14, turn)).to(BF16))
            s["res"].mul_(0.5)
            graph.replay()
            eager = step(**s)
            torch.cuda.synchronize()
            for a, b in zip(out, eager):
                assert torch.equal(a, b), turn


def test_calls_on_two_streams(device):
    states = [step_state(device, i) for i in (3, 4)]
    want = [step(**s) for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    got = [None, None]
    for _ in range(3):
        for i, (s, stream) in enumerate(zip(states, streams)):
            with torch.cuda.stream(stream):
                got[i] = step(**s)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_prompt_read_back_for_its_own_attention(device):
    """A prompt written in 8 bits and read back for sconv_diffattn_forward sees what the paged call sees of its last token."""
    g = gen(15)
    cache = filled(device, g, [90, 40], 16, 2, 32, 64, BF16, E4M3, True)
    n = torch.tensor([90, 40], dtype=torch.int32, device=device)
    k, v = sconv.sconv_cache_read(cache, 90, torch.zeros_like(n), n)
    q, lam = torch.randn(2, 1, 8, 32, generator=g).to(BF16).to(device), torch.full((4,), 0.5, device=device)
    a = sconv.sconv_diffattn_forward(q, k, v, lam, causal=True, k_lengths=n)
    b = sconv.sconv_diffattn_paged(q, cache, lam, n, causal=True)
    want, bound = attend(q, cache, lam, [90, 40], None, True)
    within(a, want, bound, "contiguous")
    within(b, want, bound, "paged")
