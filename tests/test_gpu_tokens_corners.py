"""The token operators in corners: arguments that change between calls, infinities that a query sees, angles and gradients to their last bits."""
import math

import pytest
import torch

import paper_1909_09927_amd as sconv
import tokens_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _randn(seed, *shape, dtype=F32):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


# ---- numbers given as tensors (a learned temperature): every call takes what they hold then

@pytest.mark.parametrize("where", ["cpu", "cuda"])
def test_numbers_in_tensors_are_read_at_every_call(device, where):
    q, k = _randn(1, 1, 20, 4, 32).to(device), _randn(2, 1, 20, 4, 32).to(device)
    v, lam = _randn(3, 1, 20, 2, 64).to(device), torch.tensor([0.4, 0.6], device=device)
    dout = _randn(4, 1, 20, 2, 64).to(device)
    scale, causal = torch.tensor(0.5, device=where), torch.tensor(False, device=where)

    def step(scale, causal):
        out, second, lse = sconv.sconv_diffattn_forward(q, k, v, lam, scale=scale, causal=causal, save=True)
        return (out, lse, *sconv.sconv_diffattn_backward(dout, q, k, v, lam, out, second, lse, scale=scale, causal=causal))

    for number, flag in ((0.5, False), (0.125, False), (0.125, True), (0.5, True)):
        scale.fill_(number)
        causal.fill_(flag)
        assert all(torch.equal(a, b) for a, b in zip(step(scale, causal), step(number, flag))), (number, flag)
    eps = torch.tensor(1e-5, device=where)
    for number in (1e-5, 0.5):
        eps.fill_(number)
        assert torch.equal(sconv.sconv_layernorm_forward(v, eps=eps), sconv.sconv_layernorm_forward(v, eps=number)), number


def test_rotary_axes_and_order_are_read_at_every_call(device):
    q = _randn(5, 2, 9, 2, 16).to(device)
    pos = torch.arange(18, dtype=torch.int32, device=device).view(9, 2)
    freq = torch.linspace(0.1, 1.0, 8, device=device)
    for axes in (torch.zeros(8, dtype=torch.int64), bytearray(8), [0] * 8):
        inter = torch.tensor(False)
        for p, order in ((0, False), (5, False), (7, True)):
            axes[p] = 1
            inter.fill_(order)
            got, _ = sconv.sconv_rotary_forward(q, None, pos, freq, axes, interleaved=inter)
            want, _ = sconv.sconv_rotary_forward(q, None, pos, freq, bytes(int(a) for a in axes), interleaved=order)
            assert torch.equal(got, want), (type(axes), p)
    with pytest.raises(TypeError):
        sconv.sconv_diffattn_forward(q, q, q[:, :, :1], torch.ones(1, device=device), scale="0.5")
