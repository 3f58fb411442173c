"""Performance cases of the token operators: what a network runs between its convolution stages and its answer when it
goes on with attention - layer norm (from a feature map or from tokens), rotary positions over several axes, differential
attention - forward, backward and one token at a time.

A case is a dict of plain values:
    op          "norm", "rotary" or "attention"
    dtype       "fp32" or "bf16" (norm: of x; out: of y)
    grad        norm, rotary: the backward call alone; attention: a training pass, forward and backward
  norm          layout ("map": x is [N, C, S], "tokens": x is [N, S, C]; y is [N, S, C] always), N, S, C, affine, stats (mean
                and rstd are returned, as a training program asks)
  rotary        B, S, Hq, Hk (0: queries alone), D, sections (pairs of each axis, as "28,18,18"), grid (extent of the axes,
                as "16,28,28"), interleaved, step (one token a request, each at its own place)
  attention     B, Sq, Sk, H, Hkv, D, Dv, causal, lengths (keys of request b: Sk * (b + 1) / B in some order), padded (keys are
                a grid of side x side places of which every image covers its own upper left part), side
  fused         rotary, attention: queries, keys (and values) are slices of one projection's output

Sizes are the maps of the repository's layers (VGG-19, ResNet-50, DenseNet-121, RegNetX) as tokens: 7x7 to 56x56 places of
256 to 2048 channels, up to 16 such maps in sequence, and caches of up to 32768 tokens.
"""
import math

import torch

own = False

_DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2}


def _norm(name, layout, N, S, C, dtype="bf16", out=None, grad=False, affine=True, stats=False):
    return {"name": name, "op": "norm", "layout": layout, "N": N, "S": S, "C": C, "dtype": dtype, "out": out or dtype,
            "grad": grad, "affine": affine, "stats": stats}


def _rotary(name, B, S, Hq, Hk, D, sections, grid, dtype="bf16", grad=False, interleaved=False, step=False, fused=False):
    return {"name": name, "op": "rotary", "B": B, "S": S, "Hq": Hq, "Hk": Hk, "D": D, "sections": sections, "grid": grid,
            "dtype": dtype, "grad": grad, "interleaved": interleaved, "step": step, "fused": fused}


def _attention(name, B, Sq, Sk, H, Hkv, D, Dv, dtype="bf16", grad=False, causal=False, lengths=False, padded=False,
               side=0, fused=False):
    return {"name": name, "op": "attention", "B": B, "Sq": Sq, "Sk": Sk, "H": H, "Hkv": Hkv, "D": D, "Dv": Dv,
            "dtype": dtype, "grad": grad, "causal": causal, "lengths": lengths, "padded": padded, "side": side,
            "fused": fused}


def listed():
    return [
        # the norm before the head of a batch-1 answer: the smallest call, latency of one launch
        _norm("norm-tokens-2048x49-n1", "tokens", 1, 49, 2048),
        # from the convolution stage's map to the attention block's tokens
        _norm("norm-map-256x56-n8", "map", 8, 3136, 256, dtype="fp32", out="bf16"),
        # training: the norm inside a block, gradients of tokens, weight and bias
        _norm("norm-grad-tokens-512x28-n32", "tokens", 32, 784, 512, grad=True),
        # training: the norm behind the grouped convolution stage, gradient back into the map
        _norm("norm-grad-map-896x14-n32", "map", 32, 196, 896, dtype="fp32", grad=True),
        # places of a 28x28 map, queries and keys as the projection left them
        _rotary("rotary-image-512x28-n8", 8, 784, 8, 8, 64, "16,16", "28,28", fused=True),
        # one new token for each of 64 requests over video: latency of one launch
        _rotary("rotary-step-n64", 64, 1, 16, 4, 64, "12,10,10", "16,28,28", step=True),
        # training on 16 frames in 32 bits, neighbouring elements paired
        _rotary("rotary-grad-video-16x28x28", 1, 12544, 14, 14, 64, "12,10,10", "16,28,28", dtype="fp32", grad=True,
                interleaved=True),
        # small maps in the framework's own type
        _attention("attention-fp32-896x14-n8", 8, 196, 196, 7, 7, 64, 128, dtype="fp32"),
        # images of different sizes padded to one grid
        _attention("attention-padded-1024x56-n2", 2, 3136, 3136, 8, 8, 64, 128, padded=True, side=56, fused=True),
        # serving: one token for each of 16 requests over caches of up to 32768 tokens, four query heads to a cached head
        _attention("attention-step-n16-32768", 16, 1, 32768, 16, 4, 64, 128, causal=True, lengths=True),
        # training: a block on 28x28 maps
        _attention("attention-train-512x28-n8", 8, 784, 784, 8, 8, 32, 64, grad=True),
        # the longest: 16 frames of 28x28 places, each seeing what came before
        _attention("attention-video-16x28x28", 1, 12544, 12544, 8, 4, 64, 128, causal=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _often_even(rng, lo, hi, unit):
    """A size: usually a multiple of the unit, as networks have them, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if n < unit or rng.random() < 0.25 else n // unit * unit


def _draw_norm(rng):
    while True:
        layout = rng.choice(["tokens", "map"])
        dtype = rng.choice(["fp32", "bf16"])
        out = rng.choice(["fp32", "bf16"]) if dtype == "fp32" else dtype
        if layout == "map":
            side = _log_int(rng, 7, 56)
            N, S, C = _log_int(rng, 1, 32), side * side, _often_even(rng, 16, 2048, 16)
        else:
            N, S, C = _log_int(rng, 1, 32), _log_int(rng, 1, 3136), _often_even(rng, 16, 4096, 16)
        grad = rng.random() < 0.5
        if N * S * C <= 12.8e6:
            return _norm(None, layout, N, S, C, dtype, out, grad, rng.random() < 0.8, rng.random() < 0.5)


def _draw_rotary(rng):
    while True:
        D = rng.choice([32, 64, 64, 64, 128, rng.randint(4, 60) * 2])
        pairs = D // 2 if rng.random() < 0.8 else max(1, D // 4)     # the rest of a head is left as it is
        axes = min(rng.choice([1, 2, 2, 3, 4]), pairs)
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))
        step = rng.random() < 0.3
        grid = [_log_int(rng, 1, 56) for _ in range(axes)]
        S = 1 if step else math.prod(grid)
        B = _log_int(rng, 1, 64)
        Hk = rng.choice([0, 1, 2, 4, 8, 14])
        Hq = max(Hk, 1) * rng.choice([1, 1, 2, 4])
        dtype = rng.choice(["fp32", "bf16"])
        if S <= 12544 and B * S * (Hq + Hk) * D <= 12544 * 28 * 64:
            return _rotary(None, B, S, Hq, Hk, D, sections, ",".join(map(str, grid)), dtype, rng.random() < 0.4,
                           rng.random() < 0.4, step, Hk > 0 and rng.random() < 0.5)


def _draw_attention(rng):
    while True:
        kind = rng.choice(["whole", "step", "train"])
        dtype = rng.choice(["fp32", "bf16", "bf16"])
        D = rng.choice([16, 32, 64, 64, 128, rng.randint(3, 16) * 8, rng.randint(9, 127)])
        Dv = rng.choice([2 * D, 2 * D, 2 * D, D])
        Hkv = rng.choice([1, 2, 4, 7, 8])
        H = Hkv * rng.choice([1, 1, 2, 4, 8])
        B = _log_int(rng, 1, 32)
        causal = rng.random() < 0.5
        lengths = rng.random() < 0.4
        padded, side, fused = False, 0, False
        if kind == "step":
            Sq, Sk, causal, lengths = rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 1, 32768), True, True
        else:
            # (a query that sees one key alone has no gradient: what is trained on has some)
            lo, hi = (8, 3136) if kind == "train" else (1, 12544)
            Sq = _log_int(rng, lo, hi)
            Sk = Sq if rng.random() < 0.7 else _log_int(rng, lo, hi)
            if rng.random() < 0.3:
                padded, lengths, causal, side = True, False, False, _log_int(rng, 3, 56)
                Sq = Sk = side * side
            fused = Sq == Sk and rng.random() < 0.4
        case = _attention(None, B, Sq, Sk, H, Hkv, D, Dv, dtype, kind == "train", causal, lengths, padded, side, fused)
        w = work(case)
        full = B * H * Sq * Sk * (D + Dv) * 4.0
        if kind == "train":
            full *= 2.3
        if full <= 1.9e11 * (0.25 if dtype == "fp32" else 1.0) and w["bytes"] <= 5.4e8 and B * H * Sq * Sk <= 6.0e8:
            return case


def draw(rng):
    case = rng.choice([_draw_norm, _draw_rotary, _draw_attention, _draw_attention])(rng)
    del case["name"]
    return case


def _lengths(case):
    """Keys of the requests, in rising order: spread over the whole cache."""
    B, Sk = case["B"], case["Sk"]
    return [max(1, Sk * (b + 1) // B) for b in range(B)]


def _extents(case):
    """Rows and columns of the grid that the images cover: wide ones are low."""
    B, side = case["B"], case["side"]
    return [(max(1, side * (B + b + 1) // (2 * B)), max(1, side * (2 * B - b) // (2 * B))) for b in range(B)]


def _axes(case):
    return [int(n) for n in case["sections"].split(",")]


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    dt = _DT[case["dtype"]]
    if case["op"] == "norm":
        N, S, C = case["N"], case["S"], case["C"]
        # channels with scales and means of their own, as a stage leaves them; the map carries ReLU's zeros
        centre, spread = 0.5 * randn(C), 1.0 + 0.3 * randn(C).abs()
        t = {"eps": 1e-5, "w": None, "b": None}
        if case["layout"] == "map":
            t["x"] = (randn(N, C, S) * spread[:, None] + centre[:, None]).relu_().to(dt)
        else:
            t["x"] = (randn(N, S, C) * spread + centre).to(dt)
        if case["affine"]:
            t["w"], t["b"] = 1.0 + 0.1 * randn(C), 0.1 * randn(C)
        if case["grad"]:
            t["dy"] = randn(N, S, C, dtype=_DT[case["out"]])
            xf = t["x"].float()
            dim = 1 if case["layout"] == "map" else 2
            t["mean"] = xf.mean(dim).contiguous()
            t["rstd"] = torch.rsqrt((xf - t["mean"].unsqueeze(dim)).square().mean(dim) + t["eps"]).contiguous()
        return t
    if case["op"] == "rotary":
        B, S, Hq, Hk, D = (case[k] for k in ("B", "S", "Hq", "Hk", "D"))
        sections, grid = _axes(case), [int(n) for n in case["grid"].split(",")]
        if case["fused"]:
            both = randn(B, S, Hq + Hk, D, dtype=dt)
            q, k = both[:, :, :Hq], both[:, :, Hq:]
        else:
            q = randn(B, S, Hq, D, dtype=dt)
            k = randn(B, S, Hk, D, dtype=dt) if Hk else None
        if case["step"]:
            pos = torch.stack([torch.randint(0, n, (B, 1), generator=gen, device="cuda") for n in grid], 2)
        else:
            pos = torch.cartesian_prod(*[torch.arange(n, device="cuda") for n in grid]).reshape(1, S, len(grid))
        freq = [10000.0 ** (-i / n) for n in sections for i in range(n)]
        return {"q": q, "k": k, "pos": pos.to(torch.int32).contiguous(),
                "freq": torch.tensor(freq, dtype=torch.float32, device="cuda"),
                "axes": bytes(a for a, n in enumerate(sections) for _ in range(n))}
    B, Sq, Sk, H, Hkv, D, Dv = (case[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv"))
    if case["fused"]:
        row = randn(B, Sq, 2 * H * D + 2 * Hkv * D + Hkv * Dv)
        row[:, :, :2 * H * D] *= 1.5
        row = row.to(dt)
        q = row[:, :, :2 * H * D].unflatten(2, (2 * H, D))
        k = row[:, :, 2 * H * D:2 * (H + Hkv) * D].unflatten(2, (2 * Hkv, D))
        v = row[:, :, 2 * (H + Hkv) * D:].unflatten(2, (Hkv, Dv))
    else:
        q = (1.5 * randn(B, Sq, 2 * H, D)).to(dt)
        k, v = randn(B, Sk, 2 * Hkv, D, dtype=dt), randn(B, Sk, Hkv, Dv, dtype=dt)
    t = {"q": q, "k": k, "v": v, "lam": 0.5 + 0.1 * randn(H), "len": None, "mask": None}
    order = torch.randperm(B, generator=gen, device="cuda").tolist()
    if case["lengths"]:
        n = _lengths(case)
        t["len"] = torch.tensor([n[b] for b in order], dtype=torch.int32, device="cuda")
    if case["padded"]:
        mask = torch.zeros(B, case["side"], case["side"], dtype=torch.bool, device="cuda")
        for b, (h, w) in enumerate(_extents(case)[b] for b in order):
            mask[b, :h, :w] = True
        t["mask"] = mask.reshape(B, Sk)
    if case["grad"]:
        t["dout"] = randn(B, Sq, H, Dv, dtype=dt)
    return t


def prepare(case, seed):
    return {"case": case, "t": _inputs(case, seed)}


# ---- the operators in their plain form: elementary operations in 32 bits, rounded once at the end

def _plain_norm(case, t):
    x = t["x"].float().transpose(1, 2) if case["layout"] == "map" else t["x"].float()
    out = _DT[case["out"]]
    w = 1.0 if t["w"] is None else t["w"]
    if not case["grad"]:
        mean = x.mean(2, keepdim=True)
        centred = x - mean
        rstd = torch.rsqrt((centred * centred).mean(2, keepdim=True) + t["eps"])
        y = centred * rstd * w
        if t["b"] is not None:
            y = y + t["b"]
        y = y.to(out).contiguous()
        return (y, mean.squeeze(2), rstd.squeeze(2)) if case["stats"] else y
    dy, rstd = t["dy"].float(), t["rstd"].unsqueeze(2)
    xh = (x - t["mean"].unsqueeze(2)) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(2, keepdim=True) - xh * (g * xh).mean(2, keepdim=True))
    dx = (dx.transpose(1, 2) if case["layout"] == "map" else dx).to(t["x"].dtype).contiguous()
    return (dx, (dy * xh).sum((0, 1)), dy.sum((0, 1))) if case["affine"] else dx


def _turn(x, c, s, pairs, interleaved):
    xf = x.float()
    rest = xf[..., 2 * pairs:]
    if interleaved:
        u, v = xf[..., 0:2 * pairs:2], xf[..., 1:2 * pairs:2]
        turned = torch.stack([u * c - v * s, u * s + v * c], -1).flatten(-2)
    else:
        u, v = xf[..., :pairs], xf[..., pairs:2 * pairs]
        turned = torch.cat([u * c - v * s, u * s + v * c], -1)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _plain_rotary(case, t):
    axes = torch.tensor(list(t["axes"]), device="cuda")
    pos = t["pos"].float()[:, :, axes].unsqueeze(2)
    # the frequency in two parts, so that the larger one's product with a place is exact in 32 bits
    hi = (t["freq"].view(torch.int32) & ~0xfff).view(torch.float32)
    a, b = pos * hi, pos * (t["freq"] - hi)
    c, s = a.cos() * b.cos() - a.sin() * b.sin(), a.sin() * b.cos() + a.cos() * b.sin()
    if case["grad"]:
        s = -s
    pairs = len(t["axes"])
    q = _turn(t["q"], c, s, pairs, case["interleaved"])
    return q if t["k"] is None else (q, _turn(t["k"], c, s, pairs, case["interleaved"]))


def _seen(case, t):
    """[B, 1, Sq, Sk] (or smaller, to be broadcast): which keys a query sees; None: all."""
    B, Sq, Sk = case["B"], case["Sq"], case["Sk"]
    j = torch.arange(Sk, device="cuda")
    seen = None
    if case["lengths"]:
        seen = (j < t["len"][:, None]).view(B, 1, 1, Sk)
    if case["padded"]:
        seen = t["mask"].view(B, 1, 1, Sk)
    if case["causal"]:
        i = torch.arange(Sq, device="cuda")
        last = t["len"].view(B, 1, 1, 1) if case["lengths"] else torch.full((1, 1, 1, 1), Sk, device="cuda")
        upto = j <= i.view(1, 1, Sq, 1) + last - Sq
        seen = upto if seen is None else seen & upto
    return seen


def _softmax(scores, seen):
    if seen is not None:
        scores = scores.masked_fill_(~seen, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(torch.where(total == 0.0, 1.0, total))


def _plain_attention(case, t):
    B, Sq, Sk, H, Hkv, D, Dv = (case[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv"))
    G, scale, dt = H // Hkv, 1.0 / math.sqrt(D), t["q"].dtype
    # [B, Hkv, group, Sq, .]: the query heads of a group read the same keys
    q = t["q"].float().view(B, Sq, Hkv, G, 2, D).permute(4, 0, 2, 3, 1, 5).reshape(2, B, Hkv, G * Sq, D)
    k = t["k"].float().view(B, Sk, Hkv, 2, D).permute(3, 0, 2, 1, 4).contiguous()
    v = t["v"].float().permute(0, 2, 1, 3).contiguous()
    lam = t["lam"].view(1, Hkv, G, 1, 1).expand(B, Hkv, G, Sq, 1).reshape(B, Hkv, G * Sq, 1)
    seen = _seen(case, t)
    if seen is not None:
        seen = seen.unsqueeze(2)     # [B, 1, 1, Sq, Sk] against [B, Hkv, G, Sq, Sk]

    def weights(m):
        scores = torch.matmul(q[m], k[m].transpose(2, 3)).mul_(scale).view(B, Hkv, G, Sq, Sk)
        return _softmax(scores, seen).view(B, Hkv, G * Sq, Sk)

    def heads(x, last):
        """[B, Hkv, G * Sq, last] as [B, Sq, H, last]"""
        return x.view(B, Hkv, G, Sq, last).permute(0, 3, 1, 2, 4).reshape(B, Sq, H, last)

    a1, a2 = weights(0), weights(1)
    o1, o2 = torch.matmul(a1, v), torch.matmul(a2, v)
    out = heads(o1 - lam * o2, Dv).to(dt)
    if not case["grad"]:
        return out
    do = t["dout"].float().permute(0, 2, 1, 3).reshape(B, Hkv, G * Sq, Dv)
    d1, d2 = (do * o1).sum(-1, keepdim=True), (do * o2).sum(-1, keepdim=True)
    dv = torch.matmul((a1 - lam * a2).transpose(2, 3), do)
    g = torch.matmul(do, v.transpose(2, 3))
    ds1 = a1.mul_(g - d1)
    ds2 = a2.mul_((g - d2).mul_(-lam))
    dq = torch.stack([heads(torch.matmul(ds, k[m]).mul_(scale), D) for m, ds in enumerate((ds1, ds2))], 3)
    dk = torch.stack([torch.matmul(ds.transpose(2, 3), q[m]).mul_(scale) for m, ds in enumerate((ds1, ds2))], 2)
    dlam = -d2.view(B, H, Sq).sum((0, 2))
    return {"out": out, "dq": dq.reshape(B, Sq, 2 * H, D).to(dt),
            "dk": dk.permute(0, 3, 1, 2, 4).reshape(B, Sk, 2 * Hkv, D).to(dt),
            "dv": dv.permute(0, 2, 1, 3).contiguous().to(dt), "dlam": dlam}


# ---- the framework's calls

def _own_norm(case, t):
    import paper_1909_09927_amd as sconv
    if not case["grad"]:
        return sconv.sconv_layernorm_forward(t["x"], t["w"], t["b"], eps=t["eps"], layout=case["layout"],
                                             out_dtype=_DT[case["out"]], stats=case["stats"])
    dx, dw, db = sconv.sconv_layernorm_backward(t["dy"], t["x"], t["mean"], t["rstd"], t["w"], layout=case["layout"],
                                                param_grads=case["affine"])
    return (dx, dw, db) if case["affine"] else dx


def _own_rotary(case, t):
    import paper_1909_09927_amd as sconv
    call = sconv.sconv_rotary_backward if case["grad"] else sconv.sconv_rotary_forward
    q, k = call(t["q"], t["k"], t["pos"], t["freq"], t["axes"], interleaved=case["interleaved"])
    return q if k is None else (q, k)


def _own_attention(case, t):
    import paper_1909_09927_amd as sconv
    kw = {"causal": case["causal"], "k_lengths": t["len"], "k_mask": t["mask"]}
    if not case["grad"]:
        return sconv.sconv_diffattn_forward(t["q"], t["k"], t["v"], t["lam"], **kw)
    out, second, lse = sconv.sconv_diffattn_forward(t["q"], t["k"], t["v"], t["lam"], save=True, **kw)
    dq, dk, dv, dlam = sconv.sconv_diffattn_backward(t["dout"], t["q"], t["k"], t["v"], t["lam"], out, second, lse, **kw)
    return {"out": out, "dq": dq, "dk": dk, "dv": dv, "dlam": dlam}


_PLAIN = {"norm": _plain_norm, "rotary": _plain_rotary, "attention": _plain_attention}
_OWN = {"norm": _own_norm, "rotary": _own_rotary, "attention": _own_attention}


def run(state):
    case = state["case"]
    return (_OWN if own else _PLAIN)[case["op"]](case, state["t"])


# ---- what a pass cannot do without

def _pairs(case):
    """(query, key) pairs of one head that are seen, all requests together, and the keys that anyone sees."""
    B, Sq, Sk = case["B"], case["Sq"], case["Sk"]
    if case["padded"]:
        keys = [h * w for h, w in _extents(case)]
    else:
        keys = _lengths(case) if case["lengths"] else [Sk] * B
    pairs = 0
    for n in keys:
        if not case["causal"]:
            pairs += Sq * n
        else:      # query i sees i + n - Sq + 1 keys, none where that is negative
            first = max(0, n - Sq)
            pairs += (first + n) * (n - first + 1) // 2 - (first if n >= Sq else 0)
    return pairs, sum(keys)


def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] == "norm":
        rows, C = case["N"] * case["S"], case["C"]
        if case["grad"]:
            moved = rows * C * (2 * size + _SIZE[case["out"]]) + 8 * rows + (12 * C if case["affine"] else 0)
            return {"bytes": float(moved), "flops": 12.0 * rows * C}
        moved = rows * C * (size + _SIZE[case["out"]]) + (8 * C if case["affine"] else 0) + (8 * rows if case["stats"] else 0)
        return {"bytes": float(moved), "flops": 8.0 * rows * C}
    if case["op"] == "rotary":
        elems = case["B"] * case["S"] * (case["Hq"] + case["Hk"]) * case["D"]
        pairs = sum(_axes(case))
        places = (case["B"] if case["step"] else 1) * case["S"] * len(_axes(case))
        return {"bytes": 2.0 * elems * size + 4.0 * places + 4.0 * pairs,
                "flops": 6.0 * elems / case["D"] * pairs}
    B, Sq, Sk, H, Hkv, D, Dv = (case[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv"))
    pairs, keys = _pairs(case)
    queries, values = B * Sq * 2 * H * D, B * Sq * H * Dv
    cached = keys * Hkv * (2 * D + Dv)
    flops = 4.0 * H * pairs * (D + Dv)
    moved = queries + values + cached
    if case["grad"]:
        flops += H * pairs * (8.0 * D + 4.0 * Dv)
        moved += queries + values + B * Sk * Hkv * (2 * D + Dv)
    return {"bytes": float(moved * size), "flops": flops}


# ---- the definitions in 64 bits

def _exact_norm(case, t):
    x = t["x"].double()
    if case["layout"] == "map":
        x = x.permute(0, 2, 1)
    C, one = case["C"], torch.ones(case["C"], dtype=torch.float64, device="cuda")
    w = one if t["w"] is None else t["w"].double()
    if not case["grad"]:
        mean = x.sum(-1) / C
        rstd = (((x - mean[..., None]) ** 2).sum(-1) / C + t["eps"]) ** -0.5
        y = (x - mean[..., None]) * rstd[..., None] * w + (0.0 if t["b"] is None else t["b"].double())
        return (y, mean, rstd) if case["stats"] else y
    dy, mean, rstd = t["dy"].double(), t["mean"].double()[..., None], t["rstd"].double()[..., None]
    n = (x - mean) * rstd
    u = dy * w
    dx = (u - (u @ one)[..., None] / C - n * ((u * n) @ one)[..., None] / C) * rstd
    if case["layout"] == "map":
        dx = dx.permute(0, 2, 1)
    dx = dx.contiguous()
    return (dx, torch.einsum("nsc,nsc->c", dy, n), torch.einsum("nsc->c", dy)) if case["affine"] else dx


def _exact_rotary(case, t):
    pos = t["pos"].double()
    angle = torch.stack([pos[:, :, a] * t["freq"][p].double() for p, a in enumerate(t["axes"])], -1)
    turn = torch.polar(torch.ones_like(angle), -angle if case["grad"] else angle)[:, :, None]
    pairs = len(t["axes"])

    def rotate(x):
        out = x.double().clone()
        if case["interleaved"]:
            first, second = slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)
        else:
            first, second = slice(0, pairs), slice(pairs, 2 * pairs)
        z = torch.complex(out[..., first], out[..., second]) * turn
        out[..., first], out[..., second] = z.real, z.imag
        return out

    return rotate(t["q"]) if t["k"] is None else (rotate(t["q"]), rotate(t["k"]))


def _exact_attention(case, t):
    B, Sq, Sk, H, Hkv, D, Dv = (case[k] for k in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv"))
    G, f64 = H // Hkv, torch.float64
    out = torch.zeros(B, Sq, H, Dv, dtype=f64, device="cuda")
    dq = torch.zeros(B, Sq, 2 * H, D, dtype=f64, device="cuda")
    dk = torch.zeros(B, Sk, 2 * Hkv, D, dtype=f64, device="cuda")
    dv = torch.zeros(B, Sk, Hkv, Dv, dtype=f64, device="cuda")
    dlam = torch.zeros(H, dtype=f64, device="cuda")
    places = torch.arange(Sk, device="cuda")
    for b in range(B):
        n = int(t["len"][b]) if case["lengths"] else Sk
        for h in range(H):
            g, lam = h // G, t["lam"][h].double()
            k1, k2, v = t["k"][b, :, 2 * g].double(), t["k"][b, :, 2 * g + 1].double(), t["v"][b, :, g].double()
            rows = 4096     # so many queries at a time
            for lo in range(0, Sq, rows):
                hi = min(Sq, lo + rows)
                q1, q2 = t["q"][b, lo:hi, 2 * h].double(), t["q"][b, lo:hi, 2 * h + 1].double()
                bar = (places >= n)[None, :].expand(hi - lo, Sk)
                if case["padded"]:
                    bar = bar | ~t["mask"][b][None, :]
                if case["causal"]:
                    bar = bar | (places[None, :] > torch.arange(lo, hi, device="cuda")[:, None] + (n - Sq))
                empty = bar.all(1, keepdim=True)

                def soft(q, k):
                    s = (q @ k.t() / math.sqrt(D)).masked_fill(bar, -math.inf).masked_fill(empty, 0.0)
                    return torch.softmax(s, 1).masked_fill(empty, 0.0)

                p1, p2 = soft(q1, k1), soft(q2, k2)
                out[b, lo:hi, h] = p1 @ v - lam * (p2 @ v)
                if case["grad"]:
                    do = t["dout"][b, lo:hi, h].double()
                    dp = do @ v.t()
                    dv[b, :, g] += (p1 - lam * p2).t() @ do
                    e1, e2 = (p1 * dp).sum(1, keepdim=True), (p2 * dp).sum(1, keepdim=True)
                    s1, s2 = p1 * (dp - e1) / math.sqrt(D), p2 * (dp - e2) * (-lam / math.sqrt(D))
                    dq[b, lo:hi, 2 * h], dq[b, lo:hi, 2 * h + 1] = s1 @ k1, s2 @ k2
                    dk[b, :, 2 * g] += s1.t() @ q1
                    dk[b, :, 2 * g + 1] += s2.t() @ q2
                    dlam[h] -= e2.sum()
    return {"out": out, "dq": dq, "dk": dk, "dv": dv, "dlam": dlam} if case["grad"] else out


def exact(case, seed):
    t = _inputs(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "attention": _exact_attention}[case["op"]](case, t)
