"""The serving operators in corners: scales at both ends of their range, sums that cancel, requests that are split."""
import pytest
import torch

import paper_1909_09927_amd as sconv
import serving_ref as ref
from serving_ref import E, E4M3, U, within
from test_gpu_serving import gen, operands, spread_rows

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
            within(sconv.sconv_linear8(xd, wd, out_dtype=F32), want, bound, f"scales {a}, {b}")


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
