"""Attention over a paged cache where requests are split among wavefronts and joined: tables wider than any request, so that scratch is asked for."""
import pytest
import torch

import paper_1909_09927_amd as sconv
import serving_ref as ref
import test_gpu_serving as base
from serving_ref import E, E4M3, U, within
from test_gpu_serving import attend, filled, gen, step, step_state

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
KINDS = [(F32, E4M3), (BF16, E4M3), (F32, F32), (BF16, BF16)]
KIND_IDS = ["fp32-e4m3", "bf16-e4m3", "fp32", "bf16"]


def widened(cache, positions=40000):
    """The same cache under a table with room for so many positions."""
    page = cache.k.shape[1]
    table = torch.full((cache.table.shape[0], max(-(-positions // page), cache.table.shape[1])), -1, dtype=torch.int32, device=cache.table.device)
    table[:, :cache.table.shape[1]] = cache.table
    return cache._replace(table=table)


def split(q, cache, lam, n, **kw):
    """The call, which is split; once more with scratch of NaN that ends where it may."""
    need = sconv.sconv_diffattn_paged_workspace_size(q, cache, lam, n)
    assert need > 0
    got = sconv.sconv_diffattn_paged(q, cache, lam, n, **kw)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device=q.device)
    again = sconv.sconv_diffattn_paged(q, cache, lam, n, ws=ws[:need], **kw)
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8)) and (ws[need:] == 255).all()
    return got


@pytest.mark.parametrize("dtype,kept", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("case", base.ATTN, ids=lambda c: "-".join(map(str, c[1:])) + "-n" + "_".join(map(str, c[0])))
def test_split(device, case, dtype, kept):
    lengths, Sq, H, Hkv, D, Dv, page, causal = case
    g = gen(30, *map(int, case[1:7]))
    cache = widened(filled(device, g, lengths, page, Hkv, D, Dv, dtype, kept, heads_first=(Sq + H) % 2 == 0))
    q = (1.5 * torch.randn(len(lengths), Sq, 2 * H, D, generator=g)).to(dtype).to(device)
    lam, n = 0.3 + 0.2 * torch.randn(H, generator=g).to(device), torch.tensor(lengths, dtype=torch.int32, device=device)
    want, bound = attend(q, cache, lam, lengths, None, causal)
    within(split(q, cache, lam, n, causal=causal), want, bound, "out")
    # scratch that is too small: every request is a wavefront's
    small = torch.zeros(sconv.sconv_diffattn_paged_workspace_size(q, cache, lam, n) - 16, dtype=torch.uint8, device=device)
    within(sconv.sconv_diffattn_paged(q, cache, lam, n, causal=causal, ws=small), want, bound, "out, less scratch")
    assert (small == 0).all()


#         requests, longest, H, Hkv: stretches of several units, which go on from request to request
MANY = [(70, 90, 16, 16), (66, 300, 36, 4), (300, 90, 8, 8)]


@pytest.mark.parametrize("kept", [BF16, E4M3], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 12])
@pytest.mark.parametrize("B,longest,H,Hkv", MANY)
def test_split_many_requests_a_stretch(device, B, longest, H, Hkv, page, kept):
    g = gen(31, B, H, page)
    lengths = [int(n) for n in torch.randint(0, longest, (B,), generator=g)]
    lengths[0], lengths[1], lengths[2], lengths[B // 2], lengths[B - 1] = 0, 40, 32, 700, 0
    cache = widened(filled(device, g, lengths, page, Hkv, 32, 64, BF16, kept, True))
    q, lam = torch.randn(B, 1, 2 * H, 32, generator=g).to(BF16).to(device), 0.3 + 0.2 * torch.randn(H, generator=g).to(device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    want, bound = attend(q, cache, lam, lengths, None, True)
    within(split(q, cache, lam, n, causal=True), want, bound, "out")


# (with 16 value heads a stretch has several units, with 2 it has one)
@pytest.mark.parametrize("Hkv", [2, 16])
@pytest.mark.parametrize("dtype,kept", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("page", [16, 12])
def test_split_over_pages_that_are_not_there(device, page, dtype, kept, Hkv):
    """Holes that are whole stretches, at both ends of a request and in it, and requests of nothing else."""
    g = gen(32, page, Hkv)
    lengths = [2000, 1900, 700, 1500, 90]
    cache = widened(filled(device, g, lengths, page, Hkv, 64, 128, dtype, kept, True))
    t = cache.table
    at = [p // page for p in (0, 400, 500, 1000, 1400, 1800)]
    t[0, at[0]:at[1]] = -1
    t[0, at[2]:at[3]] = 1 << 30
    t[0, at[4] + 1] = cache.k.shape[0]
    t[1, :] = -7
    t[2, 3:] = -1
    t[3, :1499 // page] = -1
    said = [2000, 1900, 700, 1500, -3]
    n = torch.tensor(said, dtype=torch.int32, device=device)
    q, lam = torch.randn(5, 2, 4 * Hkv, 64, generator=g).to(dtype).to(device), torch.full((2 * Hkv,), 0.5, device=device)
    for causal in (True, False):
        want, bound = attend(q, cache, lam, said, None, causal)
        assert torch.isfinite(want).all() and (want[[1, 4]] == 0).all()
        got = split(q, cache, lam, n, causal=causal)
        within(got, want, bound, f"out, causal {causal}")
        assert (got[[1, 4]] == 0).all()


def _exact(q, cache, lengths, b, lam, scale):
    """Request b in 64 bits, its one query, and a bound: scores of D products, sums of n terms, a weight's and the result's rounding to the type."""
    k, v, _ = ref.gathered(cache, lengths, b)
    H, D = q.shape[2] // 2, q.shape[3]
    G = H // v.shape[1]
    out, off = [], []
    for h in range(H):
        g, qd = h // G, q[b, 0].cpu().double()
        w = []
        for m in (0, 1):
            s = (k[:, 2 * g + m] * qd[2 * h + m]).sum(1) * scale
            # (an Inf of either sign, or NaN, goes on as the formula has it)
            w.append(torch.softmax(s, 0))
        l = float(lam[h])
        read = [(x[:, None] * v[:, g]).sum(0) for x in w]
        r = read[0] - l * read[1]
        mag = sum(f * (x[:, None] * v[:, g].abs()).sum(0) for f, x in zip((1.0, abs(l)), w))
        out.append(r)
        off.append(((D + 8) * E * 2 * scale * (qd[2 * h:2 * h + 2].abs().sum() * k[torch.isfinite(k)].abs().max()) + (len(k) + 60) * E) * mag + 1.01 * U[q.dtype] * r.abs())
    return torch.stack(out), torch.stack(off) + 1e-30


@pytest.mark.parametrize("Hkv", [2, 16])
@pytest.mark.parametrize("H", [2, 12], ids=["few-rows", "rows"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("page", [16, 12])
def test_split_infinities_and_nan(device, page, dtype, H, Hkv):
    """Through the join: keys of -Inf that are whole stretches of one map, a NaN in a query, Inf among the values."""
    H = H * Hkv
    g = gen(33, page, H, Hkv)
    lengths = [900, 700, 800, 600]
    cache = widened(filled(device, g, lengths, page, Hkv, 64, 128, dtype, dtype, True))
    q, lam = torch.randn(4, 1, 2 * H, 64, generator=g).abs().to(dtype), torch.full((H,), -0.5)
    q[1, 0, 3, 5] = float("nan")
    q = q.to(device)
    n = torch.tensor(lengths, dtype=torch.int32, device=device)
    table = cache.table.cpu()

    def put(t, b, p0, p1, head, d, x):
        for p in range(p0, p1):
            t[int(table[b, p // page]), p % page, head, d] = x

    # request 0: the first map's keys 0 .. 511 of key head 0 have no weight (queries are positive)
    put(cache.k, 0, 0, 512, 0, 7, -float("inf"))
    # request 2: Inf among the values, in two stretches; request 3: keys of Inf (Inf - Inf: NaN in that map, and so in the answer)
    put(cache.v, 2, 37, 38, 0, 3, float("inf"))
    put(cache.v, 2, 700, 701, 0, 9, -float("inf"))
    put(cache.k, 3, 100, 101, 2, 1, float("inf"))
    got = split(q, cache, lam.to(device), n, scale=0.125, causal=True).cpu()
    G = H // Hkv
    nan = torch.isnan(got)
    want = torch.zeros(4, H, 128, dtype=torch.float64)
    off = torch.zeros_like(want)
    for b in range(4):
        want[b], off[b] = _exact(q, cache, lengths, b, lam, 0.125)
    assert torch.equal(torch.isnan(want), nan[:, 0])
    assert nan[1, 0, 1].all() and nan[3, 0, G:2 * G].all() and int(nan.sum()) == 128 * (1 + G)
    assert (got[2, 0, :G, 3] == float("inf")).all() and (got[2, 0, :G, 9] == -float("inf")).all()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got[:, 0]))
    within(torch.where(fine, got[:, 0].double(), 0.0), torch.where(fine, want, 0.0), torch.where(fine, off, 0.0), "out")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("page", [16, 12])
def test_split_of_far_scales(device, page, dtype):
    """Values near both ends of 32 bits joined across stretches.  Scores near 0: weights near 1 part by part, whose sum of products stays in range."""
    g = gen(34, page)
    lengths = [500, 370, 490]
    cache = widened(filled(device, g, lengths, page, 2, 64, 128, dtype, E4M3, True))
    v, vs = cache.v, cache.v_scales.clone()
    small = torch.randint(1, 3, v.shape, generator=g) + 128 * torch.randint(0, 2, v.shape, generator=g)           # 2^-9, 2^-8, either sign
    large = torch.randint(0x70, 0x7f, v.shape, generator=g) + 128 * torch.randint(0, 2, v.shape, generator=g)     # 128 .. 448
    own = torch.full_like(v.view(torch.uint8), 127)
    table = cache.table.cpu()
    for b, (bytes_, scale) in enumerate(((small, 253), (large, 1), (small, 0))):
        for i, p in enumerate(table[b][:-(-lengths[b] // page)].tolist()):
            own[p] = bytes_[p].to(torch.uint8).to(device)
            vs[p] = scale or (253 if i * page < 250 else 1)            # (one end, then the other)
    cache = cache._replace(v=own.view(E4M3), v_scales=vs)
    q, lam = (0.01 * torch.randn(3, 1, 8, 64, generator=g)).to(dtype).to(device), torch.full((4,), 0.5, device=device)
    want, bound = attend(q, cache, lam, lengths, None, True)
    # an addition of the matrix pipe may take what is below the smallest normal number, 2^-126, as 0: three pieces, a term a key
    bound = bound + 3 * 500 * 1.5 * 2.0 ** -126
    within(split(q, cache, lam, torch.tensor(lengths, dtype=torch.int32, device=device), causal=True), want, bound, "out")


# ---- captured, and on two streams

def wide_state(device, seed, **kw):
    """A step's state whose attention is split: a wide table."""
    s = step_state(device, seed, **kw)
    s["cache"] = widened(s["cache"])
    q = torch.zeros(s["x"].shape[0], 1, 2 * s["H"], s["D"], dtype=BF16, device=device)
    assert sconv.sconv_diffattn_paged_workspace_size(q, s["cache"], s["lam"], s["lens"]) > 0
    return s


def test_split_steps_captured_and_replayed(device):
    """Two graphs of split steps, whose scratch is the allocator's or one's own, replayed in turn with other inputs and lengths, eager steps between."""
    states = [wide_state(device, i) for i in (41, 42)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s in states:
            step(**s)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs, lens = [], [], [s["lens"].cpu() for s in states]
    for s in states:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(**s))
        graphs.append(graph)
    for turn in range(4):
        for i, s in enumerate(states):
            s["x"].copy_(torch.randn(s["x"].shape, generator=gen(43, turn, i)).to(BF16))
            s["lens"].copy_((torch.rand(lens[i].shape, generator=gen(44, turn, i)) * (lens[i] + 1)).int())
        for graph in graphs if turn % 2 == 0 else graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        replayed = [[t.clone() for t in out] for out in outs]
        for s, out in zip(states, replayed):
            for a, b in zip(out, step(**s)):
                assert torch.equal(a, b), turn


def test_split_calls_on_two_streams(device):
    """Long requests answered on two streams at once, each call with scratch of its own."""
    calls = []
    for i in range(2):
        g = gen(45, i)
        lengths = [3000, 17, 5000, 900]
        cache = widened(filled(device, g, lengths, 16, 2, 64, 128, BF16, E4M3, True))
        q, lam = torch.randn(4, 1, 16, 64, generator=g).to(BF16).to(device), torch.full((8,), 0.4, device=device)
        n = torch.tensor(lengths, dtype=torch.int32, device=device)
        calls.append((q, cache, lam, n, attend(q, cache, lam, lengths, None, True)))
    alone = [split(*c[:4], causal=True) for c in calls]
    for c, got in zip(calls, alone):
        within(got, *c[4], "out")
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for c, stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                got.append([sconv.sconv_diffattn_paged(*c[:4], causal=True) for _ in range(8)])
        torch.cuda.synchronize()
        for outs, want in zip(got, alone):
            assert all(torch.equal(o, want) for o in outs)
