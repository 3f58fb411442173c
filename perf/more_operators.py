"""Performance cases of the serving operators: what an attention block's step in 8 bits consists of, between one token's residual
stream and the next - root-mean-square norm with the residual's addition (and its gradient, for training), 8-bit operands
with block scales and their product, a paged cache of keys and values, quantised as it is written and read back, and
differential attention of new tokens over such a cache.

A case is a dict of plain values:
    op          "norm", "project", "linear", "cache" or "attention"
    dtype       "fp32" or "bf16"
  norm          rows, C, residual ("none", "same": of x's type, "fp32": a 32-bit stream under a bf16 branch), stats (rstd is
                returned, as a training program asks), grad (the backward call alone)
  project       M, K, N: tokens into 8 bits and through 8-bit weights; norm: x + residual is normalised on the way (in front of a block),
                otherwise x goes into 8 bits as it is (behind one); residual as above
  linear        M, K, N: operands in 8 bits are in hand; dtype is the result's
  cache         B, S, Hk, D, Hv, Dv, page, stored ("same" or "e4m3"), heads_first (a page holds head after head, or slot after
                slot), before (positions in use in front of the new tokens, at most), ragged (request b has S * (b + 1) / B new tokens):
                the new tokens' keys and values are written and read back
  attention     B, Sq, Sk, H, Hkv, D, Dv, page, stored, heads_first; request b has Sk * (b + 1) / B cached tokens, in some order; causal

Values in 8 bits are e4m3, a scale for every 128 of a row (weights: for 128 x 128, cache: for every token's head) is a byte s that stands
for 2^(s - 127).  Sizes are the maps of the repository's layers (VGG-19, ResNet-50, DenseNet-121, RegNetX) as tokens, as in
operators.py: 7x7 to 56x56 places of 256 to 2048 channels, and caches of up to 32768 tokens.
"""
import math

import torch

own = False

_DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"fp32": 4, "bf16": 2, "e4m3": 1}
_EPS = 1e-6


def _norm(name, rows, C, dtype="bf16", residual="same", stats=False, grad=False):
    return {"name": name, "op": "norm", "rows": rows, "C": C, "dtype": dtype, "residual": residual, "stats": stats, "grad": grad}


def _project(name, M, K, N, dtype="bf16", norm=False, residual="same"):
    return {"name": name, "op": "project", "M": M, "K": K, "N": N, "dtype": dtype, "norm": norm, "residual": residual}


def _linear(name, M, K, N, dtype="bf16"):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "dtype": dtype}


def _cache(name, B, S, Hk, D, Hv, Dv, page, dtype="bf16", stored="e4m3", heads_first=True, before=0, ragged=False):
    return {"name": name, "op": "cache", "B": B, "S": S, "Hk": Hk, "D": D, "Hv": Hv, "Dv": Dv, "page": page, "dtype": dtype,
            "stored": stored, "heads_first": heads_first, "before": before, "ragged": ragged}


def _attention(name, B, Sq, Sk, H, Hkv, D, Dv, page, dtype="bf16", stored="e4m3", heads_first=True):
    return {"name": name, "op": "attention", "B": B, "Sq": Sq, "Sk": Sk, "H": H, "Hkv": Hkv, "D": D, "Dv": Dv, "page": page,
            "dtype": dtype, "stored": stored, "heads_first": heads_first}


def listed():
    return [
        # one token of each of 64 requests, a 32-bit residual stream under a 16-bit branch: latency of one launch
        _norm("norm-step-2048-n64", 64, 2048, residual="fp32"),
        # the norm inside a block over 32 maps of 28x28 places
        _norm("norm-tokens-512x28-n32", 25088, 512, stats=True),
        # training: its gradient, joined with the one that comes along the residual stream
        _norm("norm-grad-512x28-n32", 25088, 512, grad=True),
        # serving: in front of the attention of 64 requests' next tokens - norm, 8 bits, queries, keys and values
        _project("project-norm-2048-n64", 64, 2048, 2048, norm=True, residual="fp32"),
        # behind it, or in front of an answer: rows of eight 28x28 maps, 1000 results a row (no whole tile)
        _project("project-896x28-to-1000-n8", 6272, 896, 1000),
        # serving: the wide product of 16 tokens, bound by the weights' read
        _linear("linear-step-2048-to-8192-n16", 16, 2048, 8192),
        # prompts of 16 frames of 28x28 places: bound by the matrix pipe
        _linear("linear-2048-to-8192-16x28x28", 12544, 2048, 8192),
        # serving: one token of each of 64 requests written somewhere behind up to 8192 others
        _cache("cache-step-n64", 64, 1, 8, 64, 4, 128, 64, before=8192),
        # prompts of up to 56x56 places written, and read back for their own attention; small pages
        _cache("cache-prompt-3136-n8", 8, 3136, 8, 64, 4, 128, 16, heads_first=False, before=100, ragged=True),
        # many short requests in 16 bits, small pages as the tokens came
        _attention("paged-step-n64-784", 64, 1, 784, 8, 8, 64, 128, 16, stored="same", heads_first=False),
        # five tokens at once of two requests over 16 frames, in 32 bits; pages that end inside every tile
        _attention("paged-tokens5-fp32-n2-12544", 2, 5, 12544, 14, 7, 32, 64, 20, dtype="fp32"),
        # serving: one token of each of 16 requests over caches of up to 32768 tokens, four query heads to a cached head
        _attention("paged-step-n16-32768", 16, 1, 32768, 16, 4, 64, 128, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _often_even(rng, lo, hi, unit):
    """A size: usually a multiple of the unit, as networks have them, sometimes any number."""
    n = _log_int(rng, lo, hi)
    return n if n < unit or rng.random() < 0.25 else n // unit * unit


def _draw_norm(rng):
    while True:
        rows, C = _log_int(rng, 1, 25088), _often_even(rng, 16, 8192, 16)
        dtype = rng.choice(["fp32", "bf16", "bf16"])
        residual = rng.choice(["none", "same", "fp32"] if dtype == "bf16" else ["none", "same"])
        if rows * C <= 12.8e6:
            return _norm(None, rows, C, dtype, residual, rng.random() < 0.5, rng.random() < 0.4)


def _draw_project(rng):
    while True:
        M, K, N = _log_int(rng, 1, 12544), _often_even(rng, 16, 8192, 16), _often_even(rng, 16, 8192, 16)
        dtype = rng.choice(["fp32", "bf16", "bf16"])
        residual = rng.choice(["none", "same", "fp32"] if dtype == "bf16" else ["none", "same"])
        norm = rng.random() < 0.6
        if M * K <= 1.28e7 and M * N <= 5.2e7 and 2.0 * M * N * K <= 2.0e11:
            return _project(None, M, K, N, dtype, norm, residual if norm else "none")


def _draw_linear(rng):
    while True:
        M, K, N = _log_int(rng, 1, 25088), _often_even(rng, 16, 16384, 16), _often_even(rng, 16, 16384, 16)
        if 2.0 * M * N * K <= 4.2e11 and M * N <= 1.0e8 and M * K <= 1.0e8:
            return _linear(None, M, K, N, rng.choice(["fp32", "bf16", "bf16"]))


def _draw_page(rng):
    return rng.choice([16, 16, 32, 64, 64, 128, 256, rng.randint(1, 100)])


def _draw_head(rng):
    return rng.choice([32, 64, 64, 128, rng.randint(2, 16) * 8, rng.randint(9, 127)])


def _draw_cache(rng):
    while True:
        B, S = _log_int(rng, 1, 64), rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 1, 12544), _log_int(rng, 1, 12544)])
        Hv, D = rng.choice([1, 2, 4, 7, 8]), _draw_head(rng)
        Dv = rng.choice([2 * D, 2 * D, D])
        dtype = rng.choice(["fp32", "bf16", "bf16"])
        case = _cache(None, B, S, 2 * Hv, D, Hv, Dv, _draw_page(rng), dtype, rng.choice(["same", "e4m3", "e4m3"]), rng.random() < 0.5,
                      _log_int(rng, 1, 8192), rng.random() < 0.4)
        if B * S * Hv * (2 * D + Dv) <= 2.6e7 and B * (case["before"] + S) * Hv * (2 * D + Dv) <= 1.0e9:
            return case


def _draw_attention(rng):
    while True:
        B, Sq, Sk = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 5]), _log_int(rng, 1, 32768)
        D = _draw_head(rng)
        Dv = rng.choice([2 * D, 2 * D, 2 * D, D])
        Hkv = rng.choice([1, 2, 4, 7, 8])
        H = Hkv * rng.choice([1, 1, 2, 4, 8])
        dtype = rng.choice(["fp32", "bf16", "bf16"])
        stored = rng.choice(["same", "e4m3", "e4m3"])
        if B * Sk * Hkv * (2 * D + Dv) * _SIZE[dtype if stored == "same" else stored] <= 5.4e8 and B * Sk * Hkv * (2 * D + Dv) <= 5.4e8 and B * Sk * H * Sq <= 2.0e7:
            return _attention(None, B, Sq, Sk, H, Hkv, D, Dv, _draw_page(rng), dtype, stored, rng.random() < 0.5)


def draw(rng):
    case = rng.choice([_draw_norm, _draw_project, _draw_linear, _draw_cache, _draw_attention, _draw_attention])(rng)
    del case["name"]
    return case


# ---- 8-bit values, plainly

def _pow2(e):
    """2^e in 32 bits, exactly: integers e of -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _exponent(top):
    """The smallest e, at least -126, for which top <= 448 * 2^e."""
    m, e = torch.frexp(top)                                 # top = m 2^e, m in [1/2, 1); 448 = 7/8 * 2^9
    return torch.where(top == 0.0, -126, (e - 9 + (m > 0.875).int()).clamp_(min=-126))


def _rows_in_blocks(x):
    """[..., K] in 32 bits as [..., blocks, 128], zeros behind the last value."""
    pad = -x.shape[-1] % 128
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, 128))


def _to8_rows(x):
    """32-bit rows -> (e4m3, scale bytes of every 128)"""
    b = _rows_in_blocks(x)
    e = _exponent(b.abs().amax(-1))
    q = (b * _pow2(-e).unsqueeze(-1)).flatten(-2)[..., :x.shape[-1]].contiguous()
    return q.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _to8_blocks(w):
    """32-bit weights [N, K] -> (e4m3, scale bytes of every 128 x 128)"""
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, -K % 128, 0, -N % 128)).unflatten(0, (-1, 128)).unflatten(2, (-1, 128))
    e = _exponent(b.abs().amax((1, 3)))
    q = (b * _pow2(-e)[:, None, :, None]).flatten(2).flatten(0, 1)[:N, :K].contiguous()
    return q.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _from8_rows(q, s):
    return (_rows_in_blocks(q.float()) * _pow2(s.int() - 127).unsqueeze(-1)).flatten(-2)[..., :q.shape[-1]]


def _from8_blocks(q, s):
    e = (s.int() - 127).repeat_interleave(128, 0).repeat_interleave(128, 1)
    return q.float() * _pow2(e[:q.shape[0], :q.shape[1]])


# ---- inputs

def _lengths(case):
    B, Sk = case["B"], case["Sk"]
    return [max(1, Sk * (b + 1) // B) for b in range(B)]


def _counts(case):
    B, S = case["B"], case["S"]
    return [S * (b + 1) // B for b in range(B)] if case["ragged"] else [S] * B


def _pages(total, page, heads, width, dtype, heads_first):
    """Empty pages [total, page, heads, width]; in memory head after head or slot after slot."""
    if heads_first:
        return torch.zeros(total, heads, page, width, dtype=dtype, device="cuda").transpose(1, 2)
    return torch.zeros(total, page, heads, width, dtype=dtype, device="cuda")


def _table(gen, B, width, per, total):
    """Pages of every request, in no order: [B, width], the first per[b] of a row in use."""
    order = torch.randperm(total, generator=gen, device="cuda").int()
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :per[b]] = order[at:at + per[b]]
        at += per[b]
    return table


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device="cuda").to(dtype)

    dt = _DT[case["dtype"]]
    if case["op"] in ("norm", "project"):
        M, C = (case["rows"], case["C"]) if case["op"] == "norm" else (case["M"], case["K"])
        # channels with scales of their own, as a residual stream has them
        spread = 0.5 + randn(C).abs()
        t = {"x": (randn(M, C) * spread).to(dt), "w": 1.0 + 0.1 * randn(C), "res": None}
        rt = torch.float32 if case["residual"] == "fp32" else dt
        if case["residual"] != "none":
            t["res"] = (2.0 * randn(M, C) * spread).to(rt)
        if case["op"] == "project":
            t["w8"], t["ws"] = _to8_blocks(randn(case["N"], C) / math.sqrt(C))
        elif case["grad"]:
            total = t["x"].float() + (0.0 if t["res"] is None else t["res"].float())
            t["total"] = total.to(rt)
            t["rstd"] = torch.rsqrt(total.square().mean(1) + _EPS)
            t["dy"] = randn(M, C, dtype=dt)
            t["dtotal"] = randn(M, C, dtype=rt) if case["residual"] != "none" else None
        return t
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        # a few channels are large, as activations have them
        x = randn(M, K) * (1.0 + 9.0 * (torch.rand(K, generator=gen, device="cuda") < 0.01))
        w = randn(N, K) / math.sqrt(K)
        (x8, xs), (w8, ws) = _to8_rows(x), _to8_blocks(w)
        return {"x8": x8, "xs": xs, "w8": w8, "ws": ws}
    B, page, heads_first = case["B"], case["page"], case["heads_first"]
    kept = torch.float8_e4m3fn if case["stored"] == "e4m3" else dt
    if case["op"] == "cache":
        S, Hk, D, Hv, Dv = (case[n] for n in ("S", "Hk", "D", "Hv", "Dv"))
        counts = _counts(case)
        order = torch.randperm(B, generator=gen, device="cuda").tolist()
        counts = [counts[b] for b in order]
        starts = torch.randint(0, case["before"] + 1, (B,), generator=gen, device="cuda").tolist()
        per = [(s + n + page - 1) // page for s, n in zip(starts, counts)]
        total = sum(per) + 1                                # (the last one is nobody's)
        t = {"k": randn(B, S, Hk, D, dtype=dt), "v": randn(B, S, Hv, Dv, dtype=dt),
             "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
             "counts": torch.tensor(counts, dtype=torch.int32, device="cuda"),
             "table": _table(gen, B, (case["before"] + S + page - 1) // page, per, total - 1),
             "kp": _pages(total, page, Hk, D, kept, heads_first), "vp": _pages(total, page, Hv, Dv, kept, heads_first), "ks": None, "vs": None}
        if case["stored"] == "e4m3":
            t["ks"] = _pages(total, page, Hk, 1, torch.uint8, heads_first).squeeze(3)
            t["vs"] = _pages(total, page, Hv, 1, torch.uint8, heads_first).squeeze(3)
        return t
    Sq, Sk, H, Hkv, D, Dv = (case[n] for n in ("Sq", "Sk", "H", "Hkv", "D", "Dv"))
    lengths = _lengths(case)
    lengths = [lengths[b] for b in torch.randperm(B, generator=gen, device="cuda").tolist()]
    per = [(n + page - 1) // page for n in lengths]
    total = sum(per)
    t = {"q": (1.5 * randn(B, Sq, 2 * H, D)).to(dt), "lam": 0.5 + 0.1 * randn(H), "ks": None, "vs": None,
         "len": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "table": _table(gen, B, (Sk + page - 1) // page, per, total)}
    for name, heads, width in (("k", 2 * Hkv, D), ("v", Hkv, Dv)):
        shape = (total, heads, page, width) if heads_first else (total, page, heads, width)
        x = randn(*shape)
        if case["stored"] == "e4m3":
            e = _exponent(x.abs().amax(-1))
            x, s = x.mul_(_pow2(-e).unsqueeze(-1)), (e + 127).to(torch.uint8)
            t[name + "s"] = s.transpose(1, 2) if heads_first else s
        x = x.to(kept)
        t[name + "p"] = x.transpose(1, 2) if heads_first else x
    return t


def prepare(case, seed):
    return {"case": case, "t": _inputs(case, seed)}


# ---- the operators in their plain form: elementary operations in 32 bits, rounded once at the end

def _normalised(t):
    """(x + residual, its norm, rstd) in 32 bits"""
    total = t["x"].float() if t["res"] is None else t["x"].float() + t["res"].float()
    rstd = torch.rsqrt((total * total).mean(1, keepdim=True) + _EPS)
    return total, total * rstd * t["w"], rstd


def _plain_norm(case, t):
    if not case["grad"]:
        total, y, rstd = _normalised(t)
        out = {"y": y.to(t["x"].dtype)}
        if t["res"] is not None:
            out["total"] = total.to(t["res"].dtype)
        if case["stats"]:
            out["rstd"] = rstd.squeeze(1)
        return out
    dy, rstd = t["dy"].float(), t["rstd"].unsqueeze(1)
    u = t["total"].float() * rstd
    g = dy * t["w"]
    d = rstd * (g - u * (g * u).mean(1, keepdim=True))
    if t["dtotal"] is not None:
        d = d + t["dtotal"].float()
    out = {"dx": d.to(t["x"].dtype), "dw": (dy * u).sum(0)}
    if case["residual"] == "fp32":
        out["dres"] = d
    return out


def _plain_project(case, t):
    if case["norm"]:
        total, x, _ = _normalised(t)
    else:
        x = t["x"].float()
    y = torch.matmul(_from8_rows(*_to8_rows(x)), _from8_blocks(t["w8"], t["ws"]).t()).to(torch.bfloat16)
    return (y, total.to(t["res"].dtype)) if t["res"] is not None and case["norm"] else y


def _plain_linear(case, t):
    return torch.matmul(_from8_rows(t["x8"], t["xs"]), _from8_blocks(t["w8"], t["ws"]).t()).to(_DT[case["dtype"]])


def _bytes_of(pages):
    """8-bit pages as bytes, to be indexed."""
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _gathered(pages, scales, page, slot):
    """[B, n, heads, width] in 32 bits: the slots of the pages."""
    x = _bytes_of(pages)[page, slot]
    if scales is None:
        return x.float()
    return x.view(torch.float8_e4m3fn).float() * _pow2(scales[page, slot].int() - 127).unsqueeze(-1)


def _plain_cache(case, t):
    S, page = case["S"], case["page"]
    i = torch.arange(S, device="cuda")
    there = i < t["counts"][:, None]
    at = t["starts"][:, None] + i
    which = torch.gather(t["table"], 1, torch.div(at, page, rounding_mode="floor")).long()
    # (what is not there goes to the page that is nobody's)
    which, slot = torch.where(there, which, t["kp"].shape[0] - 1), (at % page).long()
    out = []
    for x, pages, scales in ((t["k"], t["kp"], t["ks"]), (t["v"], t["vp"], t["vs"])):
        if scales is None:
            pages[which, slot] = x
        else:
            e = _exponent(x.float().abs().amax(-1))
            q = (x.float() * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn)
            _bytes_of(pages)[which, slot] = q.view(torch.uint8)
            scales[which, slot] = (e + 127).to(torch.uint8)
        got = _gathered(pages, scales, which, slot)
        out.append(torch.where(there[:, :, None, None], got, 0.0).to(_DT[case["dtype"]]))
    return tuple(out)


def _plain_attention(case, t):
    B, Sq, Sk, H, Hkv, D, Dv, page = (case[n] for n in ("B", "Sq", "Sk", "H", "Hkv", "D", "Dv", "page"))
    G, scale = H // Hkv, 1.0 / math.sqrt(D)
    j = torch.arange(Sk, device="cuda")
    which, slot = t["table"].long()[:, torch.div(j, page, rounding_mode="floor")], (j % page).expand(B, Sk)
    k = _gathered(t["kp"], t["ks"], which, slot).view(B, Sk, Hkv, 2, D).permute(3, 0, 2, 1, 4).contiguous()
    v = _gathered(t["vp"], t["vs"], which, slot).permute(0, 2, 1, 3).contiguous()
    q = t["q"].float().view(B, Sq, Hkv, G, 2, D).permute(4, 0, 2, 3, 1, 5).reshape(2, B, Hkv, G * Sq, D)
    lam = t["lam"].view(1, Hkv, G, 1, 1).expand(B, Hkv, G, Sq, 1).reshape(B, Hkv, G * Sq, 1)
    # the last query stands at the request's last key
    upto = torch.arange(Sq, device="cuda")[:, None] + (t["len"][:, None, None] - Sq)
    seen = ((j <= upto) & (j < t["len"][:, None, None])).view(B, 1, 1, Sq, Sk)

    def read(m):
        s = torch.matmul(q[m], k[m].transpose(2, 3)).mul_(scale).view(B, Hkv, G, Sq, Sk).masked_fill_(~seen, float("-inf"))
        top = s.amax(-1, keepdim=True)
        p = s.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        return torch.matmul(p.div_(torch.where(total == 0.0, 1.0, total)).view(B, Hkv, G * Sq, Sk), v)

    out = read(0) - lam * read(1)
    return out.view(B, Hkv, G, Sq, Dv).permute(0, 3, 1, 2, 4).reshape(B, Sq, H, Dv).to(t["q"].dtype)


# ---- the framework's calls

def _own_norm(case, t):
    import paper_1909_09927_amd as sconv
    if case["grad"]:
        dx, dres, dw = sconv.sconv_rmsnorm_backward(t["dy"], t["total"], t["rstd"], t["w"], dtotal=t["dtotal"], x_dtype=t["x"].dtype)
        out = {"dx": dx, "dw": dw}
        if case["residual"] == "fp32":
            out["dres"] = dres
        return out
    y, total, rstd = sconv.sconv_rmsnorm_forward(t["x"], t["w"], residual=t["res"], eps=_EPS, stats=case["stats"])
    return {n: x for n, x in (("y", y), ("total", total), ("rstd", rstd)) if x is not None}


def _own_project(case, t):
    import paper_1909_09927_amd as sconv
    total = None
    if case["norm"]:
        x, total, _ = sconv.sconv_rmsnorm_forward(t["x"], t["w"], residual=t["res"], eps=_EPS, out_dtype=torch.float8_e4m3fn)
    else:
        x = sconv.sconv_quant8(t["x"])
    y = sconv.sconv_linear8(x, (t["w8"], t["ws"]))
    return y if total is None else (y, total)


def _own_linear(case, t):
    import paper_1909_09927_amd as sconv
    return sconv.sconv_linear8((t["x8"], t["xs"]), (t["w8"], t["ws"]), out_dtype=_DT[case["dtype"]])


def _own_cache(case, t):
    import paper_1909_09927_amd as sconv
    cache = sconv.PagedCache(t["kp"], t["vp"], t["table"], t["ks"], t["vs"])
    sconv.sconv_cache_write(cache, t["k"], t["v"], t["starts"], t["counts"])
    return sconv.sconv_cache_read(cache, case["S"], t["starts"], t["counts"], out_dtype=_DT[case["dtype"]])


def _own_attention(case, t):
    import paper_1909_09927_amd as sconv
    cache = sconv.PagedCache(t["kp"], t["vp"], t["table"], t["ks"], t["vs"])
    return sconv.sconv_diffattn_paged(t["q"], cache, t["lam"], t["len"], causal=True)


_PLAIN = {"norm": _plain_norm, "project": _plain_project, "linear": _plain_linear, "cache": _plain_cache, "attention": _plain_attention}
_OWN = {"norm": _own_norm, "project": _own_project, "linear": _own_linear, "cache": _own_cache, "attention": _own_attention}


def run(state):
    case = state["case"]
    return (_OWN if own else _PLAIN)[case["op"]](case, state["t"])


# ---- what a pass cannot do without

def _blocks(n):
    return (n + 127) // 128


def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] == "norm":
        rows, C = case["rows"], case["C"]
        stream = {"none": 0, "same": size, "fp32": 4}[case["residual"]]
        if case["grad"]:
            # dy, the sum, its gradient so far; the gradients (one where the types are one)
            moved = rows * C * (2 * size + (2 * stream if stream else size) + (stream if case["residual"] == "fp32" else 0)) + 4 * rows + 8 * C
            return {"bytes": float(moved), "flops": 10.0 * rows * C}
        return {"bytes": float(rows * C * (2 * size + 2 * stream) + 4 * C + (4 * rows if case["stats"] else 0)), "flops": 5.0 * rows * C}
    if case["op"] in ("project", "linear"):
        M, K, N = case["M"], case["K"], case["N"]
        moved = N * K + _blocks(N) * _blocks(K) + M * N * (2 if case["op"] == "project" else size)
        flops = 2.0 * M * N * K
        if case["op"] == "linear":
            moved += M * K + M * _blocks(K)
        else:
            stream = {"none": 0, "same": size, "fp32": 4}[case["residual"]] if case["norm"] else 0
            moved += M * K * (size + 2 * stream) + (4 * K if case["norm"] else 0)
            flops += (8.0 if case["norm"] else 3.0) * M * K
        return {"bytes": float(moved), "flops": flops}
    one = _SIZE["e4m3"] if case["stored"] == "e4m3" else size
    if case["op"] == "cache":
        tokens, values = sum(_counts(case)), case["Hk"] * case["D"] + case["Hv"] * case["Dv"]
        scales = 2 * (case["Hk"] + case["Hv"]) if case["stored"] == "e4m3" else 0
        # rows that are not there are read back as zeros
        moved = tokens * (values * (size + 2 * one) + scales) + case["B"] * case["S"] * values * size
        return {"bytes": float(moved), "flops": 4.0 * tokens * values}
    B, Sq, H, Hkv, D, Dv = (case[n] for n in ("B", "Sq", "H", "Hkv", "D", "Dv"))
    lengths = _lengths(case)
    pairs = sum(sum(max(0, n - i) for i in range(Sq)) for n in lengths)
    moved = B * Sq * H * (2 * D + Dv) * size + sum(lengths) * Hkv * ((2 * D + Dv) * one + (3 if case["stored"] == "e4m3" else 0))
    moved += 4 * sum((n + case["page"] - 1) // case["page"] for n in lengths)
    return {"bytes": float(moved), "flops": 4.0 * H * pairs * (D + Dv)}


# ---- the definitions in 64 bits

def _grid8(x, dims):
    """x in 64 bits as its 8-bit form holds it, a scale over `dims`: from the format's definition (three bits behind the leading one,
    the smallest step 2^-9, nothing above 448; half a step goes to the even neighbour)."""
    top = x.abs().amax(dims, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0)).clamp(min=-126.0)       # (of 0: -Inf)
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1.0, e)
    e = torch.where((top <= 448.0 * torch.exp2(e - 1.0)) & (e > -126.0), e - 1.0, e)
    v = x / torch.exp2(e)
    lead = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    lead = torch.where(torch.exp2(lead + 1.0) <= v.abs(), lead + 1.0, lead)
    step = torch.exp2(lead - 3.0)
    return torch.round(v / step) * step * torch.exp2(e)


def _grid8_rows(x):
    K = x.shape[-1]
    b = torch.cat([x, x.new_zeros(*x.shape[:-1], -K % 128)], -1).reshape(*x.shape[:-1], -1, 128)
    return _grid8(b, -1).reshape(*x.shape[:-1], -1)[..., :K]


def _exact_norm(case, t):
    total = t["x"].double() + (0.0 if t["res"] is None else t["res"].double())
    if not case["grad"]:
        rstd = (total.pow(2).sum(1) / case["C"] + _EPS) ** -0.5
        out = {"y": total * rstd[:, None] * t["w"].double()}
        if t["res"] is not None:
            out["total"] = total
        if case["stats"]:
            out["rstd"] = rstd
        return out
    rstd, dy = t["rstd"].double(), t["dy"].double()
    n = t["total"].double() * rstd[:, None]
    g = dy * t["w"].double()
    d = (g - n * ((g * n).sum(1) / case["C"])[:, None]) * rstd[:, None]
    if t["dtotal"] is not None:
        d += t["dtotal"].double()
    out = {"dx": d, "dw": torch.einsum("rc,rc->c", dy, n)}
    if case["residual"] == "fp32":
        out["dres"] = d
    return out


def _exact_project(case, t):
    x = t["x"].double()
    total = x + (0.0 if t["res"] is None or not case["norm"] else t["res"].double())
    if case["norm"]:
        x = total * ((total.pow(2).sum(1) / case["K"] + _EPS) ** -0.5)[:, None] * t["w"].double()
    y = _grid8_rows(x) @ _weights(t).t()
    return (y, total) if t["res"] is not None and case["norm"] else y


def _weights(t):
    N, K = t["w8"].shape
    n, k = torch.arange(N, device="cuda") // 128, torch.arange(K, device="cuda") // 128
    return t["w8"].double() * 2.0 ** (t["ws"].double() - 127.0)[n][:, k]


def _exact_linear(case, t):
    k = torch.arange(case["K"], device="cuda") // 128
    x = t["x8"].double() * 2.0 ** (t["xs"].double() - 127.0)[:, k]
    return x @ _weights(t).t()


def _exact_cache(case, t):
    there = torch.arange(case["S"], device="cuda") < t["counts"][:, None]
    out = []
    for x in (t["k"].double(), t["v"].double()):
        if case["stored"] == "e4m3":
            x = _grid8(x, -1)
        out.append(x * there[:, :, None, None])
    return tuple(out)


def _exact_attention(case, t):
    B, Sq, H, Hkv, D, Dv, page = (case[n] for n in ("B", "Sq", "H", "Hkv", "D", "Dv", "page"))
    out = torch.zeros(B, Sq, H, Dv, dtype=torch.float64, device="cuda")
    for b, n in enumerate(t["len"].tolist()):
        used = t["table"][b, :(n + page - 1) // page].long()

        def of(pages, scales):
            x = pages[used].double() if scales is None else pages.view(torch.uint8)[used].view(torch.float8_e4m3fn).double()
            if scales is not None:
                x = x * 2.0 ** (scales[used].double() - 127.0)[..., None]
            return x.flatten(0, 1)[:n]

        k, v = of(t["kp"], t["ks"]), of(t["vp"], t["vs"])
        hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n - Sq, n, device="cuda")[:, None]
        empty = hidden.all(1, keepdim=True)
        for h in range(H):
            g = h // (H // Hkv)

            def soft(m):
                s = (t["q"][b, :, 2 * h + m].double() @ k[:, 2 * g + m].t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
                return torch.softmax(s.masked_fill(empty, 0.0), 1).masked_fill(empty, 0.0) @ v[:, g]

            out[b, :, h] = soft(0) - t["lam"][h].double() * soft(1)
    return out


def exact(case, seed):
    t = _inputs(case, seed)
    return {"norm": _exact_norm, "project": _exact_project, "linear": _exact_linear, "cache": _exact_cache,
            "attention": _exact_attention}[case["op"]](case, t)
