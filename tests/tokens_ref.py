"""Plain token operators in 64 bits on the CPU, each with a bound on what a computation in a given type may be off by.

U[type] is the type's unit roundoff; sums of n terms in 32 bits are within n * 2^-24 of their absolute terms.  Bounds are built
from the inputs alone, before any result is looked at.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
E = 2.0 ** -24


def norm(x, w, b, eps, out_dtype):
    """x [..., C] -> (y, mean, rstd), bound of y, bound of mean, bound of rstd"""
    x = x.double()
    C = x.shape[-1]
    w = torch.ones(C, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(C, dtype=torch.float64) if b is None else b.double()
    mean = x.mean(-1, keepdim=True)
    var = (x - mean).square().mean(-1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    y = (x - mean) * rstd * w + b
    # sums: at most C / 16 terms in a lane's own order, never more than 300, and 8 steps over lanes
    n = min(C, 300) + 12
    off = n * E * x.abs().mean(-1, keepdim=True)                   # of the mean
    rel = n * E + off * rstd + (off * rstd) ** 2                   # of rstd: half its square's relative error, twice as much here
    by = (off * rstd + (x - mean).abs() * rstd * (rel + 4 * E)) * w.abs() + 2 * E * b.abs() + U[out_dtype] * y.abs() * 1.01
    return (y, mean.squeeze(-1), rstd.squeeze(-1)), (by + 1e-30, off.squeeze(-1) + 1e-30, (rel * rstd).squeeze(-1))


def norm_grad(dy, x, mean, rstd, w):
    """-> (dx, dw, db), their bounds (32-bit sums; the types' own rounding apart)"""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double().unsqueeze(-1), rstd.double().unsqueeze(-1)
    C = x.shape[-1]
    w = torch.ones(C, dtype=torch.float64) if w is None else w.double()
    u = (x - mean) * rstd
    # (x - mean in 32 bits: one rounding of the difference)
    bu = 2 * E * u.abs() + E * (x - mean).abs() * rstd
    g = dy * w
    m1, m2 = g.mean(-1, keepdim=True), (g * u).mean(-1, keepdim=True)
    dx = rstd * (g - m1 - u * m2)
    n = min(C, 300) + 16
    b1 = n * E * g.abs().mean(-1, keepdim=True)
    b2 = n * E * (g * u).abs().mean(-1, keepdim=True) + (g.abs() * bu).mean(-1, keepdim=True)
    bx = rstd * (4 * E * (g.abs() + m1.abs() + (u * m2).abs()) + b1 + u.abs() * b2 + bu * m2.abs())
    lead = tuple(range(x.dim() - 1))
    rows = min(x[..., 0].numel(), 700) + 16
    dw, db = (dy * u).sum(lead), dy.sum(lead)
    bw = rows * E * (dy * u).abs().sum(lead) + (dy.abs() * bu).sum(lead)
    return (dx, dw, db), (bx + 1e-30, bw + 1e-30, rows * E * dy.abs().sum(lead) + 1e-30)


def rotary(x, pos, freq, axes, interleaved, inverse):
    """x [B, S, H, D], pos [B or 1, S, A] -> (y, bound apart from y's rounding)"""
    pairs = len(axes)
    x, y = x.double(), x.double().clone()
    t = torch.stack([pos[:, :, a].double() * freq[p].double() for p, a in enumerate(axes)], -1).unsqueeze(2)
    c, s = t.cos(), (-t.sin() if inverse else t.sin())
    i = slice(0, 2 * pairs, 2) if interleaved else slice(0, pairs)
    j = slice(1, 2 * pairs, 2) if interleaved else slice(pairs, 2 * pairs)
    u, v = x[..., i], x[..., j]
    y[..., i], y[..., j] = u * c - v * s, u * s + v * c
    bound = torch.zeros_like(x)
    # cosine and sine are within 2^-23 (argument, polynomial), then two products and a sum
    bound[..., i] = bound[..., j] = 5 * E * (u.abs() + v.abs())
    return y, bound + 1e-30


def visible(B, Sq, Sk, causal, lengths, mask):
    """[B, Sq, Sk]"""
    j = torch.arange(Sk)
    n = torch.full((B,), Sk) if lengths is None else lengths.long().clamp(0, Sk)
    seen = (j < n[:, None])[:, None, :].expand(B, Sq, Sk)
    if causal:
        seen = seen & (j <= (torch.arange(Sq)[:, None] + n[:, None, None] - Sq))
    if mask is not None:
        seen = seen & mask.bool()[:, None, :]
    return seen


def attention(q, k, v, lam, scale, causal, lengths, mask, dout=None):
    """Differential attention head by head: a dict of results and a dict of their bounds."""
    dt = q.dtype
    u = U[dt]
    B, Sq, H2, D = q.shape
    Sk, Hkv, Dv = k.shape[1], v.shape[2], v.shape[3]
    H = H2 // 2
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    seen = visible(B, Sq, Sk, causal, lengths, mask)
    f64 = torch.float64
    z = lambda *s: torch.zeros(*s, dtype=f64)  # noqa: E731
    r = {"out": z(B, Sq, H, Dv), "second": z(B, Sq, H, Dv), "lse": z(2, B, H, Sq)}
    e = {n: z(*t.shape) for n, t in r.items()}
    if dout is not None:
        for n, s in (("dq", q.shape), ("dk", k.shape), ("dv", v.shape), ("dlam", lam.shape)):
            r[n], e[n] = z(*s), z(*s)
    for b in range(B):
        # keys that are left out are never part of a sum; what causal alone hides has to be finite
        there = seen[b].any(0) if Sq else torch.zeros(Sk, dtype=torch.bool)
        for h in range(H):
            g = h // (H // Hkv)
            l = float(lam[h])
            K = [torch.where(there[:, None], k[b, :, 2 * g + m].double(), 0.0) for m in (0, 1)]
            V = torch.where(there[:, None], v[b, :, g].double(), 0.0)
            some = seen[b].any(1, keepdim=True)
            Q = [torch.where(some, q[b, :, 2 * h + m].double(), 0.0) for m in (0, 1)]
            A, EA = [], []
            for m in (0, 1):
                s = (Q[m] @ K[m].t()) * scale
                mag = (Q[m].abs() @ K[m].abs().t()) * scale
                s = s.masked_fill(~seen[b], -math.inf)
                p = torch.softmax(s.masked_fill(~some, 0.0), 1).masked_fill(~some, 0.0)
                # a weight: its score and the scores its sum stands on, exp2 and its argument, the sum
                worst = (mag * seen[b]).amax(1, keepdim=True) if Sk else z(Sq, 1)
                A.append(p)
                EA.append(p * ((D + 8) * E * (mag + worst) + (min(Sk, 700) + 40) * E))
                lse = torch.logsumexp(s, 1) if Sk else torch.full((Sq,), -math.inf, dtype=f64)
                r["lse"][m, b, h] = lse
                e["lse"][m, b, h] = (D + 8) * E * worst[:, 0] + (min(Sk, 700) + 40) * E + 4 * E * torch.where(lse.isfinite(), lse, 0.0).abs()
            # each map's weights are rounded to the type for their product with the values, which sums in 32 bits
            part = [(EA[m] + (1.01 * u + (Sk + 8) * E) * A[m]) @ V.abs() for m in (0, 1)]
            O = [A[m] @ V for m in (0, 1)]
            r["out"][b, :, h], r["second"][b, :, h] = O[0] - l * O[1], O[1]
            e["out"][b, :, h] = part[0] + abs(l) * part[1] + 1.01 * u * (O[0] - l * O[1]).abs()
            e["second"][b, :, h] = part[1] + 1.01 * u * O[1].abs()
            if dout is None:
                continue
            dO = torch.where(some, dout[b, :, h].double(), 0.0)
            G = dO @ V.t()
            EG = (Dv + 4) * E * (dO.abs() @ V.abs().t())
            P = A[0] - l * A[1]
            EP = EA[0] + abs(l) * EA[1] + 2 * E * (A[0] + abs(l) * A[1]) + 1.01 * u * P.abs()
            r["dv"][b, :, g] += P.t() @ dO
            e["dv"][b, :, g] += (EP + (H // Hkv * Sq + 8) * E * P.abs()).t() @ dO.abs()
            # d_m from the results as they were rounded
            sums = (Dv + 8) * E
            ed2 = (dO.abs() * e["second"][b, :, h]).sum(1, keepdim=True) + sums * (dO * O[1]).abs().sum(1, keepdim=True)
            ed1 = (dO.abs() * e["out"][b, :, h]).sum(1, keepdim=True) + abs(l) * ed2 + sums * (dO.abs() * (O[0].abs() + 2 * abs(l) * O[1].abs())).sum(1, keepdim=True)
            for m, (c, ed) in enumerate(((1.0, ed1), (-l, ed2))):
                d = (A[m] * G).sum(1, keepdim=True)
                S = c * A[m] * (G - d)
                ES = abs(c) * (EA[m] * (G - d).abs() + A[m] * (EG + ed + 4 * E * (G.abs() + d.abs()))) + 1.01 * u * S.abs()
                r["dq"][b, :, 2 * h + m] = scale * (S @ K[m])
                e["dq"][b, :, 2 * h + m] = scale * ((ES + (Sk + 8) * E * S.abs()) @ K[m].abs())
                r["dk"][b, :, 2 * g + m] += scale * (S.t() @ Q[m])
                e["dk"][b, :, 2 * g + m] += scale * ((ES + (H // Hkv * Sq + 8) * E * S.abs()).t() @ Q[m].abs())
            r["dlam"][h] -= (A[1] * G).sum()
            e["dlam"][h] += (EA[1] * G.abs() + A[1] * (EG + (min(Sk, 700) + min(B * Sq, 700) + 40) * E * G.abs())).sum()
    for n in ("dq", "dk", "dv"):
        if n in r:
            e[n] += 1.01 * u * r[n].abs()
    return r, {n: t + 1e-30 for n, t in e.items()}


def within(got, want, bound, what):
    """Every value within its bound of the wanted one; infinities equal."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)}, not {tuple(want.shape)}"
    same = got == want
    off = (got - want).abs()
    bad = ~same & ~(off <= bound)
    if bad.any():
        at = torch.nonzero(bad)[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {at}: {got[tuple(at)].item()} for "
                             f"{want[tuple(at)].item()}, bound {bound[tuple(at)].item() if bound.shape == want.shape else bound}")
