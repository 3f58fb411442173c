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


# ---- infinities that a query sees: what the formulas make of them

SHAPES = [(1, 40, 50, 2, 1, 64, 128), (1, 1, 300, 4, 2, 64, 128), (2, 150, 97, 2, 2, 72, 144), (1, 33, 70, 1, 1, 128, 256), (1, 1, 1, 1, 1, 32, 64),
          (1, 130, 200, 1, 1, 32, 64)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_visible_minus_infinity_key_has_no_weight(device, shape, dtype):
    """Scores of -Inf: the key counts for nothing, as if it were not there.  Queries of few bits (1, 1.5), whose lower parts are zero, and
    of many."""
    B, Sq, Sk, H, Hkv, D, Dv = shape
    q, k, v = _randn(11, B, Sq, 2 * H, D, dtype=dtype), _randn(12, B, Sk, 2 * Hkv, D, dtype=dtype), _randn(13, B, Sk, Hkv, Dv, dtype=dtype)
    lam = 0.5 + 0.1 * _randn(14, H)
    q[..., 3] = torch.tensor([1.0, 1.5, 0.1, 2.0 ** -20]).to(dtype)[torch.arange(q[..., 3].numel()) % 4].view(q.shape[:-1])
    gone = torch.zeros(B, Sk, dtype=torch.bool)
    gone[:, Sk // 2] = gone[:, Sk - 1] = True
    clean = k.clone()
    k[gone] = k[gone].index_fill(2, torch.tensor([3]), -math.inf)
    r, e = ref.attention(q, clean, v, lam, None, False, None, ~gone)
    out, second, lse = sconv.sconv_diffattn_forward(q.to(device), k.to(device), v.to(device), lam.to(device), save=True)
    for name, got in (("out", out), ("second", second), ("lse", lse)):
        ref.within(got, r[name], e[name], name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention_visible_infinite_value(device, shape, dtype):
    """A column of V with an Inf: Inf in that column of every result (lam below 0, so that the maps' parts have one sign), the other columns
    as they are."""
    B, Sq, Sk, H, Hkv, D, Dv = shape
    q, k, v = _randn(15, B, Sq, 2 * H, D, dtype=dtype), _randn(16, B, Sk, 2 * Hkv, D, dtype=dtype), _randn(17, B, Sk, Hkv, Dv, dtype=dtype)
    lam = -0.5 - 0.1 * _randn(18, H).abs()
    r, e = ref.attention(q, k, v, lam, None, False, None, None)
    v[:, Sk // 2, :, 5], v[:, Sk // 2, :, 9] = math.inf, -math.inf
    out, second, _ = sconv.sconv_diffattn_forward(q.to(device), k.to(device), v.to(device), lam.to(device), save=True)
    for name, got in (("out", out), ("second", second)):
        for c, s in ((5, math.inf), (9, -math.inf)):
            r[name][..., c] = s
        ref.within(got, r[name], e[name], name)


def test_attention_infinite_scores_and_their_rows(device):
    """+Inf among a row's scores, and 0 * Inf in one: that row is NaN and no other."""
    for dtype in (F32, BF16):
        q, k, v = _randn(21, 1, 64, 2, 64, dtype=dtype), _randn(22, 1, 90, 2, 64, dtype=dtype), _randn(23, 1, 90, 1, 128, dtype=dtype)
        q[..., 3] = 1.0
        k[:, 7, :, 3] = -math.inf
        q[0, 10, :, 3], q[0, 40, :, 3] = -1.0, 0.0
        out = sconv.sconv_diffattn_forward(q.to(device), k.to(device), v.to(device), torch.full((1,), 0.5, device=device)).cpu()
        bad = out[0].isnan().flatten(1).all(1)
        assert bad.nonzero().flatten().tolist() == [10, 40] and out[0, ~bad].isfinite().all()


def test_attention_gradient_that_overflows(device):
    """dout V^T beyond 32 bits under weights of a half: dS is Inf, and dq = Inf times keys of one sign each, not NaN."""
    D, Dv, H = 16, 32, 1
    q, k, v = torch.zeros(1, 3, 2, D), torch.ones(1, 2, 2, D), torch.zeros(1, 2, 1, Dv)
    k[0, 1] = -1.0
    v[0, 0], v[0, 1] = 3e38, -3e38
    lam, dout = torch.tensor([-1.0]), torch.full((1, 3, 1, Dv), 2.0)
    dev = [t.to(device) for t in (q, k, v, lam)]
    out, second, lse = sconv.sconv_diffattn_forward(*dev, save=True)
    assert not out.any() and not second.any()
    dq = sconv.sconv_diffattn_backward(dout.to(device), *dev, out, second, lse)[0]
    assert (dq == math.inf).all()


# ---- the last bits

@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_cosine_is_centred(device, interleaved):
    """Cosines short of an eighth of a turn, where a polynomial cut off too early is off to one side.  Each of the 11200 is within about 2^-24, in
    either direction by its roundings: their mean is within 2^-24 / 100 of 0 then, and 2^-28 is asked for."""
    pairs, pos = 8, torch.arange(49900, 51300, dtype=torch.int32).view(1, -1, 1)
    freq = 2.0 ** -16 * (1.0 + torch.arange(pairs) * 2.0 ** -13)
    x = torch.zeros(1, pos.shape[1], 1, 2 * pairs)
    first = slice(0, None, 2) if interleaved else slice(0, pairs)
    x[..., first] = 1.0
    y, _ = sconv.sconv_rotary_forward(x.to(device), None, pos.to(device), freq.to(device), bytes(pairs), interleaved=interleaved)
    off = y.cpu().double()[..., first] - (pos.double() * freq.double()).cos().unsqueeze(2)
    assert off.abs().max() <= 2.0 ** -23 and abs(off.mean()) <= 2.0 ** -28


@pytest.mark.parametrize("shape", [(2, 1, 900, 4, 2, 64, 128), (1, 1, 70, 2, 2, 32, 64), (1, 4, 300, 8, 1, 64, 128), (2, 3, 400, 2, 1, 61, 122),
                                   (1, 5, 500, 10, 2, 128, 256), (1, 8, 300, 4, 1, 100, 37)], ids=str)
def test_attention_of_few_rows_is_rounded_once(device, shape):
    """16-bit results of up to 32 rows a key head: as far off as the exact ones rounded to 16 bits are, to a twentieth (weights to 2^-16, 32-bit
    sums; weights to 2^-8 would add as much again)."""
    B, Sq, Sk, H, Hkv, D, Dv = shape
    q, k, v = 1.5 * _randn(41, B, Sq, 2 * H, D), _randn(42, B, Sk, 2 * Hkv, D, dtype=BF16), _randn(43, B, Sk, Hkv, Dv, dtype=BF16)
    q, lam = q.to(BF16), 0.5 + 0.1 * _randn(44, H)
    r, _ = ref.attention(q, k, v, lam, None, True, None, None)
    got = sconv.sconv_diffattn_forward(q.to(device), k.to(device), v.to(device), lam.to(device), causal=True, save=True)
    for name, t in zip(("out", "second"), got):
        own = (r[name].to(BF16).double() - r[name]).norm()
        assert (t.cpu().double() - r[name]).norm() <= 1.05 * own, name


@pytest.mark.parametrize("D", [32, 64])
def test_attention_gradients_are_near_their_rounding(device, D):
    """16-bit dq and dk over 784 places: their own rounding is 1.66e-3 of their norm, d_m from rounded results brings dq to 1.9e-3.  With dS rounded
    to 16 bits alone, instead of going as two values, dq is 2.5e-3 (64) and 2.6e-3 (32) off."""
    S, H = 784, 2
    q, k, v = (1.5 * _randn(31, 2, S, 2 * H, D)).to(BF16), _randn(32, 2, S, 2 * H, D, dtype=BF16), _randn(33, 2, S, H, 2 * D, dtype=BF16)
    dout, lam = _randn(34, 2, S, H, 2 * D, dtype=BF16), 0.5 + 0.1 * _randn(35, H)
    r, _ = ref.attention(q, k, v, lam, None, False, None, None, dout)
    dev = [t.to(device) for t in (q, k, v, lam)]
    grads = sconv.sconv_diffattn_backward(dout.to(device), *dev, *sconv.sconv_diffattn_forward(*dev, save=True))
    for name, got in zip(("dq", "dk"), grads):
        off = (got.cpu().double() - r[name]).norm() / r[name].norm()
        assert off <= 2.2e-3, (name, float(off))
