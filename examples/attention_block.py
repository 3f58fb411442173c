"""An attention block behind a convolution stage: how the convolution calls and the token operators go together.

    map [N, C, H, W]  --sconv_forward (3x3, ReLU)-->  map
                      --sconv_layernorm (map to tokens)-->  tokens [N, H*W, C]
                      --projection-->  queries, keys, values (slices of one tensor)
                      --sconv_rotary (rows and columns of the map)-->  queries, keys
                      --sconv_diffattn-->  heads  --sconv_layernorm (every head)-->  projection, back onto the map

`forward` answers, `forward(..., save=True)` and `backward` train, and `look` asks one token a request over the keys and values of
the frames seen so far (a video): positions then have three axes.  Projections are torch's matrix products.

    python examples/attention_block.py        # a stage of 256 channels on 28x28 maps, timed
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1909_09927_amd as sconv  # noqa: E402


class AttentionBlock:
    def __init__(self, channels, heads, key_heads=None, head=32, dtype=torch.bfloat16, lam_init=0.2, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def randn(*shape):
            return torch.randn(shape, generator=g, device=device)

        self.C, self.H, self.Hkv, self.D, self.dtype, self.lam_init = channels, heads, key_heads or heads, head, dtype, lam_init
        rows = 2 * heads * head + self.Hkv * 4 * head              # queries, keys (two each), values of twice a head's width
        self.conv = randn(channels, channels, 3, 3) * math.sqrt(2.0 / (9 * channels))
        self.norm_w, self.norm_b = torch.ones(channels, device=device), torch.zeros(channels, device=device)
        self.head_w = torch.ones(2 * head, device=device)
        self.w_in = (randn(rows, channels) / math.sqrt(channels)).to(dtype)
        self.w_out = (randn(channels, heads * 2 * head) / math.sqrt(heads * 2 * head)).to(dtype)
        self.lam_vectors = 0.1 * randn(4, heads, head)             # of every head: lam = exp(a . b) - exp(c . d) + lam_init
        n = head // 4                                              # pairs of an axis: rows and columns share a head
        self.axes = sconv.sconv_rotary_axes((n, head // 2 - n))
        self.freq = torch.tensor([100.0 ** (-i / n) for n in (n, head // 2 - n) for i in range(n)], device=device)

    def lam(self):
        a, b, c, d = self.lam_vectors
        return ((a * b).sum(1).exp() - (c * d).sum(1).exp() + self.lam_init).contiguous()

    @staticmethod
    def places(H, W, device="cuda"):
        """Positions of a map's places: row and column."""
        return torch.cartesian_prod(torch.arange(H, device=device), torch.arange(W, device=device)).to(torch.int32)

    def _project(self, tokens):
        """Queries, keys and values as slices of the projection's output."""
        row = tokens @ self.w_in.t()
        a, b = 2 * self.H * self.D, 2 * (self.H + self.Hkv) * self.D
        return (row[..., :a].unflatten(-1, (2 * self.H, self.D)), row[..., a:b].unflatten(-1, (2 * self.Hkv, self.D)),
                row[..., b:].unflatten(-1, (self.Hkv, 2 * self.D)))

    def _finish(self, heads, save):
        """Every head normalised, the heads projected onto channels: [N, C, places]."""
        out = sconv.sconv_layernorm_forward(heads, self.head_w, stats=save)
        y, stats = (out[0], out[1:]) if save else (out, None)
        flat = y.flatten(2) * (1.0 - self.lam_init)
        return torch.matmul(self.w_out, flat.transpose(1, 2).contiguous()).float(), flat, stats

    def forward(self, x, k_mask=None, save=False):
        """map -> map; save: (map, what backward reads).  k_mask: [N, H*W], false at places that are padding."""
        stage = sconv.sconv_forward(x, self.conv, 1, 1, relu=True)
        N, C, H, W = stage.shape
        out = sconv.sconv_layernorm_forward(stage, self.norm_w, self.norm_b, layout="map", out_dtype=self.dtype, stats=save)
        tokens, stats = (out[0], out[1:]) if save else (out, None)
        q, k, v = self._project(tokens)
        pos = self.places(H, W, x.device)
        q, k = sconv.sconv_rotary_forward(q, k, pos, self.freq, self.axes)
        lam = self.lam()
        got = sconv.sconv_diffattn_forward(q, k, v, lam, k_mask=k_mask, save=save)
        heads, second, lse = got if save else (got, None, None)
        add, flat, head_stats = self._finish(heads, save)
        y = stage + add.view_as(stage)
        if not save:
            return y
        return y, dict(stage=stage, tokens=tokens, stats=stats, q=q, k=k, v=v, pos=pos, lam=lam, heads=heads, second=second, lse=lse, flat=flat,
                       head_stats=head_stats, k_mask=k_mask)

    def backward(self, dy, s):
        """Gradients of the stage's map and of the block's weights (the convolution's filters stay as they are)."""
        N, C, H, W = dy.shape
        add = dy.view(N, C, H * W).transpose(1, 2).to(self.dtype).contiguous()              # of every place
        dw_out = torch.matmul(add.flatten(0, 1).t(), s["flat"].flatten(0, 1))
        dflat = (add @ self.w_out) * (1.0 - self.lam_init)
        dheads, dhead_w, _ = sconv.sconv_layernorm_backward(dflat.view_as(s["heads"]), s["heads"], *s["head_stats"], self.head_w)
        dq, dk, dv, dlam = sconv.sconv_diffattn_backward(dheads, s["q"], s["k"], s["v"], s["lam"], s["heads"], s["second"], s["lse"],
                                                         k_mask=s["k_mask"])
        dq, dk = sconv.sconv_rotary_backward(dq, dk, s["pos"], self.freq, self.axes, out=(dq, dk))
        drow = torch.cat([dq.flatten(2), dk.flatten(2), dv.flatten(2)], 2)
        dw_in = torch.matmul(drow.flatten(0, 1).t(), s["tokens"].flatten(0, 1))
        dtokens = drow @ self.w_in
        dstage, dnorm_w, dnorm_b = sconv.sconv_layernorm_backward(dtokens, s["stage"], *s["stats"], self.norm_w, layout="map")
        a, b, c, d = self.lam_vectors
        first, second = ((a * b).sum(1).exp() * dlam)[:, None], ((c * d).sum(1).exp() * dlam)[:, None]
        return {"stage": dstage + dy, "norm_w": dnorm_w, "norm_b": dnorm_b, "w_in": dw_in, "w_out": dw_out, "head_w": dhead_w,
                "lam_vectors": torch.stack([first * b, first * a, -second * d, -second * c])}

    # ---- one token a request over the frames seen so far

    def cache(self, requests, capacity, device="cuda"):
        n = 2 * self.Hkv * self.D
        return {"k": torch.empty(requests, capacity, 2 * self.Hkv, self.D, dtype=self.dtype, device=device),
                "v": torch.empty(requests, capacity, self.Hkv, n // self.Hkv, dtype=self.dtype, device=device),
                "len": torch.zeros(requests, dtype=torch.int32, device=device)}

    def video_axes(self):
        n = self.D // 8
        sections = (n, n, self.D // 2 - 2 * n)
        freq = torch.tensor([100.0 ** (-i / s) for s in sections for i in range(s)], device=self.freq.device)
        return sconv.sconv_rotary_axes(sections), freq

    def remember(self, cache, tokens, frame, H, W):
        """Appends a frame's keys and values, all requests in step: tokens [requests, H*W, C]."""
        _, k, v = self._project(tokens)
        places = self.places(H, W, tokens.device)
        pos = torch.cat([torch.full_like(places[:, :1], frame), places], 1).contiguous()
        axes, freq = self.video_axes()
        k, _ = sconv.sconv_rotary_forward(k, None, pos, freq, axes)
        at = int(cache["len"][0])
        cache["k"][:, at:at + H * W], cache["v"][:, at:at + H * W] = k, v
        cache["len"] += H * W

    def look(self, cache, token, pos):
        """What one token of every request ([requests, 1, C], at [requests, 1, 3]) sees: [requests, 1, heads * 2 * head]."""
        q, _, _ = self._project(token)
        axes, freq = self.video_axes()
        q, _ = sconv.sconv_rotary_forward(q, None, pos, freq, axes)
        heads = sconv.sconv_diffattn_forward(q, cache["k"], cache["v"], self.lam(), causal=True, k_lengths=cache["len"])
        return sconv.sconv_layernorm_forward(heads, self.head_w).flatten(2) * (1.0 - self.lam_init)


def main():
    block, x = AttentionBlock(256, 4), torch.randn(8, 256, 28, 28, device="cuda").relu_()
    y, saved = block.forward(x, save=True)
    dy = torch.randn_like(y)
    cache = block.cache(8, 16 * 784)
    for frame in range(16):
        block.remember(cache, saved["tokens"], frame, 28, 28)
    pos = torch.tensor([15, 27, 27], dtype=torch.int32, device="cuda").expand(8, 1, 3).contiguous()

    def timed(what, f, n=20):
        for _ in range(3):
            f()
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        for _ in range(n):
            f()
        e[1].record()
        torch.cuda.synchronize()
        print(f"{what}: {e[0].elapsed_time(e[1]) / n * 1e3:.0f} us")

    timed("8 maps of 256 x 28 x 28, forward", lambda: block.forward(x))
    timed("  forward and backward", lambda: block.backward(dy, block.forward(x, save=True)[1]))
    timed("one token of 8 requests over 16 frames (12544 keys)", lambda: block.look(cache, saved["tokens"][:, -1:].contiguous(), pos))


if __name__ == "__main__":
    main()
