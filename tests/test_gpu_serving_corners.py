"""The serving operators in corners: scales at both ends of their range, sums that cancel, requests that are split."""
import pytest
import torch

import paper_1909_09927_amd as sconv
import serving_ref as ref
from serving_ref import E, E4M3, U, within
from test_gpu_serving import gen, new_cache, operands, spread_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


# ---- the product: scales at the ends of their range

def _small_bytes(shape, g):
    """2^-9 .. 3 * 2^-9, either sign."""
    return (torch.randint(1, 4, shape, generator=g) + 128 * torch.randint(0, 2, shape, generator=g)).to(torch.uint8).view(E4M3)


def _product(x, w, dtype):
    """In 64 bits, and a bound: sums in 32 bits, one rounding to the type; where a block's two partial sums are scaled below the smallest
    normal number each is rounded to a whole multiple of 2^-149."""
    (xq, xs), (wq, ws) = x, w
    a, b = ref.held(xq, xs), ref.held(wq, ws, 128)
    want, K = a @ b.t(), a.shape[1]
    off = (K + 16) * E * (a.abs() @ b.abs().t()) + 1.01 * U[dtype] * want.abs() + (2 * xs.shape[1] + 1) * 2.0 ** -150
    return want, off + (2.0 ** -134 if dtype == BF16 else 0.0)


def _both(x, w, device):
    """The operands on the device at whole vectors, and at no aligned address."""
    yield tuple((q.to(device), s.to(device)) for q, s in (x, w))
    yield tuple((spread_rows(q.view(torch.uint8), device).view(E4M3), s.to(device)) for q, s in (x, w))


# (4096 x 4096: tiles of 256 x 256)
FAR = [(5, 20, 256), (64, 150, 300), (65, 150, 300), (300, 300, 400), (4096, 4096, 256)]
#      scales of x and of w, w's values small: products of 2^-180 to 2^128
ENDS = [(60, 60, False), (1, 120, False), (120, 1, False), (50, 60, False), (10, 100, False), (70, 75, False), (127, 246, True), (246, 127, True), (185, 187, True), (254, 118, True)]


@pytest.mark.parametrize("M,N,K", FAR)
def test_linear8_of_products_at_both_ends(device, M, N, K):
    """Results are the formula's wherever 32 bits hold them, whichever operand's scales take them there."""
    g = gen(20, M, K)
    (xq, xs), (wq, ws) = operands(M, N, K, g)
    tiny = _small_bytes(wq.shape, g)
    for a, b, small in ENDS if M < 4096 else ((60, 60, False), (127, 246, True)):
        xs.fill_(a)
        ws.fill_(b)
        x, w = (xq, xs), (tiny if small else wq, ws)
        want, bound = _product(x, w, F32)
        assert (want != 0).any() and want.abs().max() < 3e38
        for xd, wd in _both(x, w, device):
            y = sconv.sconv_linear8(xd, wd, out_dtype=F32)
            within(y, want, bound, f"scales {a}, {b}")
            assert torch.equal(sconv.sconv_linear8(xd, wd, exact=True), y.to(BF16)), f"scales {a}, {b}, rounded"


@pytest.mark.parametrize("M,N,K", FAR)
def test_linear8_of_scales_of_every_size(device, M, N, K):
    """Far rows and blocks beside ordinary ones, blocks of zeros with the smallest scale, NaN in a far row."""
    g = gen(21, M, K)
    (xq, xs), (wq, ws) = operands(M, N, K, g)
    xs[:] = torch.randint(20, 161, xs.shape, generator=g).to(torch.uint8)
    ws[:] = torch.tensor([60, 190], dtype=torch.uint8).repeat(1, ws.shape[1])[:, :ws.shape[1]]
    xq.view(torch.uint8)[M // 2, :128] = 0
    xs[M // 2, 0] = 1
    wq.view(torch.uint8)[:min(N, 128), 128:] = 128                     # (-0)
    ws[0, 1:] = 1
    want, bound = _product((xq, xs), (wq, ws), F32)
    for xd, wd in _both((xq, xs), (wq, ws), device):
        within(sconv.sconv_linear8(xd, wd, out_dtype=F32), want, bound, "y")
    xq.view(torch.uint8)[1, 5] = 0x7f
    xs[1, 0] = 3
    for xd, wd in _both((xq, xs), (wq, ws), device):
        y = sconv.sconv_linear8(xd, wd, out_dtype=F32).cpu()
        assert torch.isnan(y[1]).all()
        keep = torch.arange(M) != 1
        within(y[keep], want[keep], bound[keep], "rows beside a NaN")


@pytest.mark.parametrize("M,N", [(65, 150), (4096, 4100)])
def test_linear8_of_a_far_block_behind_ordinary_ones(device, M, N):
    """The last of 122 blocks (more than a tile's scales in LDS are read at once) is far; tiles of rows without it are not."""
    K = 122 * 128 if M < 4096 else 256
    g = gen(22, M)
    (xq, xs), (wq, ws) = operands(M, N, K, g)
    xs[:, :-1], xs[:, -1], ws[:, -1] = 60, 50, 50
    xs[40:] = 127
    ws[:, :-1] = 100
    want, bound = _product((xq, xs), (wq, ws), F32)
    for xd, wd in _both((xq, xs), (wq, ws), device):
        within(sconv.sconv_linear8(xd, wd, out_dtype=F32), want, bound, "y")


# ---- the product: 16-bit results by exact products, and by the matrix pipe's 8-bit ones

def _cancelling(M, N, K, g):
    """Two channels of 1000 times the rest, whose products take each other away but for their rounding to 8 bits."""
    x, w = torch.randn(M, K, generator=g), torch.randn(N, K, generator=g)
    x[:, 5], x[:, K - 9], w[:, K - 9] = 1000.0, -1000.0, w[:, 5]
    return [(torch.from_numpy(q).view(E4M3), torch.from_numpy(s)) for q, s in (ref.quant8(x), ref.quant8(w, 128))]


SHAPES = [(3, 40, 256), (17, 300, 256), (64, 300, 256), (33, 4200, 130), (65, 300, 256), (300, 300, 2048), (4096, 4096, 256)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear8_exact(device, M, N, K):
    """16-bit results that are the 32-bit ones rounded once, where products cancel and where they do not; of up to 64 rows always."""
    for x, w in (_cancelling(M, N, K, gen(23, M)), operands(M, N, K, gen(24, M))):
        want, bound = _product(x, w, BF16)
        for xd, wd in _both(x, w, device):
            y = sconv.sconv_linear8(xd, wd, exact=True)
            assert y.dtype == BF16
            within(y, want, bound, "y")
            assert torch.equal(y, sconv.sconv_linear8(xd, wd, out_dtype=F32).to(BF16))
            assert torch.equal(y, sconv.sconv_linear8(xd, wd, exact=torch.ones(1, device=device)))
            if M <= 64:
                assert torch.equal(y, sconv.sconv_linear8(xd, wd))


@pytest.mark.parametrize("M,N,K", [(65, 1024, 512), (100, 4200, 512), (1024, 1024, 2048), (4096, 4096, 512)])
def test_linear8_cuts_off_no_more_than_is_said(device, M, N, K):
    """The matrix pipe's products of normal values against the 64-bit result rounded once, as a whole and in every row and column.  An error d moves a
    rounding to its neighbour, one step away, with a chance of |d| / step, so the squares of what moves add up to |d| * step each, and a step
    is at most 2^-7 of a value: d of 1.4e-5 of the norm moves sqrt(2^-7 * 1.4e-5) = 3.4e-4 of it.  A row has at least 1024 values, of which a
    dozen move: three times as much by chance."""
    g = gen(25, M, K)
    x, w = torch.randn(M, K, generator=g), torch.randn(N, K, generator=g)
    x, w = [(torch.from_numpy(q).view(E4M3), torch.from_numpy(s)) for q, s in (ref.quant8(x), ref.quant8(w, 128))]
    want = ref.held(*x) @ ref.held(*w, 128).t()
    for xd, wd in _both(x, w, device):
        off = sconv.sconv_linear8(xd, wd).cpu().double() - want.to(BF16).double()
        said = 3.4e-4
        assert off.norm() <= said * want.norm()
        assert (off.norm(dim=1) <= 3 * said * want.norm(dim=1)).all()
        if M >= 1024:
            assert (off.norm(dim=0) <= 3 * said * want.norm(dim=0)).all()


@pytest.mark.parametrize("M,N,K", [(65, 150, 300), (300, 300, 400), (4096, 4096, 256)])
def test_linear8_by_the_pipe_at_far_scales_and_outliers(device, M, N, K):
    """Each result within the bound that the format's cut gives: less than 2^-10 of the product of the largest magnitudes of every eight depths, of which
    those without a leading one (2^-6 of the scale) may count as 2^-6; what is below the smallest normal number may be taken as 0."""
    g = gen(26, M, K)
    (xq, xs), (wq, ws) = operands(M, N, K, g)
    tiny = _small_bytes(wq.shape, g)
    k = torch.arange(K) // 128
    cases = [((xq, xs.clone().fill_(a)), (tiny if small else wq, ws.clone().fill_(b))) for a, b, small in (ENDS if M < 4096 else ENDS[:1])]
    for x, w in cases + [_cancelling(M, N, K, g)]:
        want, bound = _product(x, w, BF16)
        tops = [ref._tops_of_eight(ref.held(q, s, rows), 2.0 ** (s.double() - 133.0)[torch.arange(q.shape[0]) // rows][:, k]) for (q, s), rows in ((x, 1), (w, 128))]
        bound = bound + 2.0 ** -10 * (tops[0] @ tops[1].t()) + (K // 8 + 1) * 2.0 ** -126
        for xd, wd in _both(x, w, device):
            within(sconv.sconv_linear8(xd, wd), want, bound, f"scales {int(x[1][0, 0])}, {int(w[1][0, 0])}")


# ---- attention: weights of 32 bits

def _written(device, k, v, page, kept):
    """A cache that holds keys [B, n, 2Hkv, D] and values [B, n, Hkv, Dv], and its lengths."""
    B, n = k.shape[:2]
    cache = new_cache(device, gen(27, page), B, [-(-n // page)] * B, page, k.shape[2], k.shape[3], v.shape[2], v.shape[3], kept, True)
    lengths = torch.full((B,), n, dtype=torch.int32, device=device)
    sconv.sconv_cache_write(cache, k.to(device), v.to(device), torch.zeros_like(lengths))
    return cache, lengths


@pytest.mark.parametrize("H", [4, 24], ids=["few-rows", "rows"])
@pytest.mark.parametrize("kept", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 12])
@pytest.mark.parametrize("D,Dv", [(64, 128), (32, 64), (40, 72)])
def test_paged_weights_of_two_keys_that_cancel(device, D, Dv, page, kept, H):
    """Two keys of nearly equal weights whose values are 1 and -1: what is left is 2^-8 and less, and shows what weights are rounded to.

    A weight's argument: the score is one exact product of at most 2^-8, its factor is rounded twice, the difference with the largest once: below E.  Its
    exponential: 2 E.  The sum of two, their quotient and the products' sums of two: 2 E, 2 E, 4 E, and the two maps' difference 2 E: 12 E of either map."""
    B, Hkv = 64, 2
    g = gen(28, D, H)
    k, v = torch.zeros(B, 2, 2 * Hkv, D), torch.ones(B, 2, Hkv, Dv)
    k[:, 0, :, 0], k[:, 1, :, 0], v[:, 1] = 1.0, -1.0, -1.0
    q = torch.zeros(B, 1, 2 * H, D)
    q[..., 0] = 2.0 ** -8 * (2.0 * torch.rand(B, 1, 2 * H, generator=g) - 1.0)
    q, lam = q.to(BF16), -torch.rand(H, generator=g)
    cache, n = _written(device, k.to(BF16), v.to(BF16), page, kept)
    got = sconv.sconv_diffattn_paged(q.to(device), cache, lam.to(device), n, scale=1.0).cpu().double()
    left = torch.tanh(q[..., 0].double()).view(B, 1, H, 2)             # (e^s - e^-s) / (e^s + e^-s)
    l = lam.double()
    want = (left[..., 0] - l * left[..., 1]).unsqueeze(-1).expand(B, 1, H, Dv)
    within(got, want, 12 * E * (1.0 + l.abs())[:, None] + 1.01 * U[BF16] * want.abs(), "out")


@pytest.mark.parametrize("H", [4, 24], ids=["few-rows", "rows"])
@pytest.mark.parametrize("page", [16, 12])
def test_paged_values_of_infinity(device, page, H):
    """An Inf among the values is its column's answer whatever its weight, 1 and other powers of two among them; other columns do not see it."""
    B, n, Hkv, D, Dv = 3, 32, 2, 64, 128
    g = gen(29, H)
    k, v = torch.zeros(B, n, 2 * Hkv, D), torch.randn(B, n, Hkv, Dv, generator=g)
    k[1, :, :, 0] = -torch.arange(n)[:, None].float()
    k[2] = torch.randn(n, 2 * Hkv, D, generator=g)
    v = v.to(BF16)
    v[:, 5, 1, 7], v[:, 0, 1, 9], v[:, 20, 0, 100] = float("inf"), float("inf"), -float("inf")
    q = torch.randn(B, 1, 2 * H, D, generator=g)
    q[1] = 0.0
    q[1, :, :, 0] = 1.0
    cache, lengths = _written(device, k.to(BF16), v, page, BF16)
    lam = torch.full((H,), -0.5, device=device)
    got = sconv.sconv_diffattn_paged(q.to(BF16).to(device), cache, lam, lengths, scale=0.6931471805599453).cpu()
    G = H // Hkv
    assert (got[:, 0, G:, 7] == float("inf")).all() and (got[:, 0, G:, 9] == float("inf")).all() and (got[:, 0, :G, 100] == -float("inf")).all()
    keep = torch.ones(H, Dv, dtype=torch.bool)
    keep[G:, 7] = keep[G:, 9] = keep[:G, 100] = False
    assert torch.isfinite(got[:, 0][:, keep]).all()


# ---- numbers given as tensors: every call takes what they hold then

@pytest.mark.parametrize("where", ["cpu", "cuda"])
def test_whole_numbers_in_tensors_are_read_at_every_call(device, where):
    cache = sconv.sconv_cache_new(2, 4, 8, 16, 2, 8, 1, 8, dtype=F32, device=device)
    cache.table.copy_(torch.arange(8, dtype=torch.int32).view(2, 4))
    k, v = torch.randn(2, 40, 2, 8, generator=gen(30)).to(device), torch.randn(2, 40, 1, 8, generator=gen(31)).to(device)
    starts = torch.zeros(2, dtype=torch.int32, device=device)
    sconv.sconv_cache_write(cache, k, v, starts)
    x = torch.randn(130, 200, generator=gen(32)).to(device)
    S, rows = torch.tensor(3, device=where), torch.tensor(1, device=where)
    for n, block in ((3, 1), (40, 128), (1, 1), (40, 128)):
        S.fill_(n)
        rows.fill_(block)
        rk, rv = sconv.sconv_cache_read(cache, S, starts)
        assert torch.equal(rk, k[:, :n]) and torch.equal(rv, v[:, :n])
        for got, want in zip(sconv.sconv_quant8(x, rows), sconv.sconv_quant8(x, block)):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
    for bad in (2.0, "3", None):
        with pytest.raises(TypeError):
            sconv.sconv_cache_read(cache, bad, starts)


# ---- refusals

def test_rmsnorm_backward_takes_what_the_forward_call_gives(device):
    """dy of y's types: bf16 anywhere, fp32 where x is fp32."""
    t = torch.randn(3, 40, generator=gen(33)).to(device)
    rstd = torch.ones(3, device=device)
    for total, dy, x_dtype, goes in ((F32, F32, None, True), (F32, F32, F32, True), (F32, BF16, None, True), (F32, BF16, BF16, True), (BF16, BF16, None, True), (BF16, BF16, BF16, True),
                                     (F32, F32, BF16, False), (BF16, F32, None, False), (BF16, F32, BF16, False), (BF16, BF16, F32, False)):
        def call():
            return sconv.sconv_rmsnorm_backward(t.to(dy), t.to(total), rstd, x_dtype=x_dtype)

        if goes:
            assert call()[0].dtype == (total if x_dtype is None else x_dtype)
        else:
            with pytest.raises(sconv.SconvError):
                call()


def test_scratch_on_another_device_is_refused(device):
    """(asked as the calls ask: of scratch on this device for tensors that are on the next)"""
    from paper_1909_09927_amd.tokens import _ws
    ws = torch.empty(64, dtype=torch.uint8, device=device)
    assert _ws(ws, 16, ws.device)[2] == 64
    with pytest.raises(ValueError):
        _ws(ws, 16, torch.device("cuda", ws.device.index + 1))
