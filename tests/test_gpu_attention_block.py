"""The attention block of examples/ against the same block in 64 bits with torch's own gradients."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _turn(x, pos, freq, axes):
    p = len(axes)
    t = torch.stack([pos[..., a].double() * freq[i].double() for i, a in enumerate(axes)], -1).unsqueeze(-2)
    u, v = x[..., :p], x[..., p:2 * p]
    return torch.cat([u * t.cos() - v * t.sin(), u * t.sin() + v * t.cos(), x[..., 2 * p:]], -1)


def _norm(x, w, b=0.0, eps=1e-5):
    m = x.mean(-1, keepdim=True)
    return (x - m) / ((x - m).square().mean(-1, keepdim=True) + eps).sqrt() * w + b


def _attend(q, k, v, lam, seen):
    """q [N, S, 2H, D], k [N, T, 2G, D], v [N, T, G, E] -> [N, S, H, E]"""
    out, H = [], q.shape[2] // 2
    for h in range(H):
        g = h // (H // v.shape[2])
        a = [torch.softmax((q[:, :, 2 * h + m] @ k[:, :, 2 * g + m].transpose(1, 2) / math.sqrt(q.shape[3])).masked_fill(~seen, -math.inf), 2)
             for m in (0, 1)]
        out.append((a[0] - lam[h] * a[1]) @ v[:, :, g])
    return torch.stack(out, 2)


def _lam(block, vectors):
    a, b, c, d = vectors
    return (a * b).sum(1).exp() - (c * d).sum(1).exp() + block.lam_init


def _split(block, row):
    a, b = 2 * block.H * block.D, 2 * (block.H + block.Hkv) * block.D
    return (row[..., :a].unflatten(-1, (2 * block.H, block.D)), row[..., a:b].unflatten(-1, (2 * block.Hkv, block.D)),
            row[..., b:].unflatten(-1, (block.Hkv, 2 * block.D)))


def _plain(block, p, mask):
    N, C, H, W = p["stage"].shape
    tokens = _norm(p["stage"].flatten(2).transpose(1, 2), p["norm_w"], p["norm_b"])
    q, k, v = _split(block, tokens @ p["w_in"].t())
    pos = block.places(H, W, "cpu")[None]
    q, k = (_turn(t, pos, block.freq.cpu(), block.axes) for t in (q, k))
    heads = _attend(q, k, v, _lam(block, p["lam_vectors"]), mask[:, None, :])
    flat = _norm(heads, p["head_w"]).flatten(2) * (1.0 - block.lam_init)
    return p["stage"] + (flat @ p["w_out"].t()).transpose(1, 2).reshape(N, C, H, W)


def _near(got, want, tol, what):
    off = (got.detach().cpu().double() - want).norm() / want.norm()
    assert off <= tol, f"{what}: {float(off):.2e} of its norm away, {tol:.0e} allowed"


# 32 bits: a dozen steps, each within some ten roundings (2^-24) of its operands; 16 bits: as many roundings to 2^-8, of random signs
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 4e-2)], ids=["fp32", "bf16"])
@pytest.mark.parametrize("channels,heads,key_heads,head,side", [(64, 2, 2, 32, 9), (96, 4, 2, 16, 7)])
def test_block(device, channels, heads, key_heads, head, side, dtype, tol):
    from attention_block import AttentionBlock
    block = AttentionBlock(channels, heads, key_heads, head, dtype=dtype, seed=3)
    g = torch.Generator()
    g.manual_seed(4)
    x, dy = torch.randn(2, channels, side, side, generator=g).relu().to(device), torch.randn(2, channels, side, side, generator=g)
    mask = torch.ones(2, side, side, dtype=torch.bool)
    mask[1, side - 2:], mask[1, :, side - 3:] = False, False
    mask = mask.flatten(1)
    y, saved = block.forward(x, mask.to(device), save=True)
    assert torch.equal(y, block.forward(x, mask.to(device)))
    got = block.backward(dy.to(device), saved)
    names = ("stage", "norm_w", "norm_b", "w_in", "w_out", "head_w", "lam_vectors")
    p = {n: (saved["stage"] if n == "stage" else getattr(block, n)).detach().cpu().double().requires_grad_() for n in names}
    want = _plain(block, p, mask)
    _near(y, want.detach(), tol, "map")
    want.backward(dy.double())
    for n in names:
        _near(got[n], p[n].grad, 3 * tol, n)


def test_one_token_over_frames(device):
    from attention_block import AttentionBlock
    block = AttentionBlock(64, 4, 2, 16, dtype=torch.float32, seed=5)
    g = torch.Generator()
    g.manual_seed(6)
    frames = torch.randn(3, 2, 20, 64, generator=g)
    cache = block.cache(2, 100)
    for t, tokens in enumerate(frames):
        block.remember(cache, tokens.to(device), t, 4, 5)
    token, pos = torch.randn(2, 1, 64, generator=g), torch.tensor([[[2, 3, 4]], [[2, 0, 1]]], dtype=torch.int32)
    got = block.look(cache, token.to(device), pos.to(device))
    axes, freq = block.video_axes()
    w = block.w_in.cpu().double()
    rows = [_split(block, f.double() @ w.t()) for f in frames]
    places = block.places(4, 5, "cpu")
    k = torch.cat([_turn(r[1], torch.cat([torch.full_like(places[:, :1], t), places], 1)[None], freq.cpu(), axes) for t, r in enumerate(rows)], 1)
    v = torch.cat([r[2] for r in rows], 1)
    q = _turn(_split(block, token.double() @ w.t())[0], pos, freq.cpu(), axes)
    heads = _attend(q, k, v, block.lam().cpu().double(), torch.ones(1, 1, 60, dtype=torch.bool))
    _near(got, _norm(heads, block.head_w.cpu().double()).flatten(2) * (1.0 - block.lam_init), 2e-5, "seen")
