"""The attention's backward passes over so many rows that their sums would lose bits if they were kept in one place of the tensor cores, which cut off."""
import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb
from test_gpu_attn_bwd import make, run_bwd, tiles_of
from test_gpu_bwd_calls import forward, sampled

pytestmark = pytest.mark.gpu


def check(name, got, want):
    """Sums of one sign that grow evenly.  A step of the tensor cores adds 16 products to a sum and cuts off less than 2^-22 of what it is by then, on
    average half of what it is in the end; after 2048 steps the sum is added to others in fp32.  So less than 2^-12 of the sum, and half a step of
    bf16 at its place: 2^-8 of the power of two below it."""
    half = torch.exp2(torch.floor(torch.log2(want)) - 8)
    over = ((got.double() - want).abs() - half) / want
    assert over.max().item() <= 2.0 ** -12, (name, over.max().item())


LONG = [(16, 1, 65536, 64), (8, 1, 49000, 128), (4, 1, 50001, 256), (6, 2, 16385, 64), (3, 1, 8193, 128)]


@pytest.mark.parametrize("Hq,Hkv,n,D,softcap,gate", [(*x, 0.0, gate) for x in LONG for gate in (False, True)] + [(2, 1, 33000, 128, 30.0, False)])
def test_sums_of_one_sign(Hq, Hkv, n, D, softcap, gate):
    """x = 0 and lse = 0, so p = 1; delta = -1 and v = 0, so ds = 1: dv, dk and dq are plain sums of do, q and k, worked out here in 64 bits"""
    G = Hq // Hkv
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    size = lambda H: (1 + 0.25 * torch.rand((1, H, n, D), generator=gen, device="cuda")).to(torch.bfloat16)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 1, n, 1.0, softcap)
    how = dict(g=torch.zeros((1, n, 4), device="cuda"), lam=1.0) if gate else {}
    zeros = torch.zeros((1, Hkv, n, D), dtype=torch.bfloat16, device="cuda")
    t = {"do": size(Hq), "v": zeros, "lse": torch.zeros((1, Hq, n), device="cuda")}
    t["do"][..., 0] = 1
    t["o"] = torch.zeros_like(t["do"])
    t["o"][..., 0] = -1
    q, k = size(Hq), size(Hkv)
    # with keys of 0, then with queries of 0
    got = run_bwd(shape, dict(t, q=q, k=zeros), **how)
    for name, x in (("dv", t["do"]), ("dk", q)):
        want = x.double().unflatten(1, (Hkv, G)).sum(2).flip(2).cumsum(2).flip(2)
        check(name, got[name], want)
    got = run_bwd(shape, dict(t, q=torch.zeros_like(q), k=k), **how)
    want = k.double().cumsum(2)
    for h in range(Hq):
        check("dq", got["dq"][:, h], want[:, h // G])


@pytest.mark.parametrize("masks", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_parts_of_ordinary_sums(D, masks):
    """16 query heads on one KV head, four of them an item: up to 300 tiles, with parts that end anywhere among the heads (and, with masks, among the tiles that are
    left out); the same bits twice, and each result near the one from heads of their own, whose items are short"""
    n, G = 9700, 16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D)
    rnd = lambda H: torch.randn((1, H, n, D), generator=gen, device="cuda").to(torch.bfloat16)
    t = {"q": rnd(G), "k": rnd(1), "v": rnd(1), "do": rnd(G)}
    # (as many KV heads as query heads: one head's items are 76 tiles at most)
    apart = dict(t, k=t["k"].expand(1, G, n, D).contiguous(), v=t["v"].expand(1, G, n, D).contiguous())
    one, many = fb.make_shape(G, 1, n, D, 8, 1, 64), fb.make_shape(G, G, n, D, 8, 1, 64)
    args, more = {}, {}
    if masks:
        m = (1 << torch.randint(0, 8, (n // 300 + 1,), generator=gen, device="cuda")).to(torch.int32).repeat_interleave(300)[:n]
        for how, s, H in ((args, one, 1), (more, many, G)):
            mq, mk = m.expand(1, G, n).contiguous(), m.expand(1, H, n).contiguous()
            tiles = fb.alloc_workspace(s, 0)
            fb.focus_build_tiles(s, mq, mk, 0, tiles)
            how.update(mq=mq, mk=mk, tiles=tiles)
    o, lse = torch.empty_like(t["q"]), torch.empty((1, G, n), device="cuda")
    fb.focus_attn_fwd(one, t["q"], t["k"], t["v"], args.get("mq"), args.get("mk"), args.get("tiles"), 0, o, lse)
    for x in (t, apart):
        x.update(o=o, lse=lse)
    a, b, c = run_bwd(one, t, **args), run_bwd(one, t, **args), run_bwd(many, apart, **more)
    assert all(torch.equal(a[x], b[x]) for x in a) and torch.equal(a["dq"], c["dq"])
    for x in ("dk", "dv"):
        # (each of the 16 summands rounded to bf16 there, the sum here)
        want, size = c[x].double().sum(1), c[x].double().abs().sum(1)
        assert ((a[x][:, 0].double() - want).abs() <= 2.0 ** -8 * size + 2.0 ** -8 * want.abs() + 2.0 ** -12 * size.max()).all(), x


@pytest.mark.parametrize("n,D,G", [(70000, 64, 1), (66000, 128, 2), (33000, 256, 1)])
def test_pieces_without_a_pair(n, D, G):
    """32 groups, each of one stretch of tokens only: most items have no pair at all in a later piece of their columns"""
    t, gen = make(1, G, 1, n, D, 1)
    m = torch.ones(1, dtype=torch.int32, device="cuda") << (torch.arange(n, device="cuda") // (n // 32 + 1)).to(torch.int32)
    mq, mk = m.expand(1, G, n).contiguous(), m.expand(1, 1, n).contiguous()
    shape = fb.make_shape(G, 1, n, D, 32, 1, 100)
    tiles = tiles_of(shape, mq, mk)
    forward(shape, t, mq, mk, tiles)
    got = run_bwd(shape, t, mq, mk, tiles)
    pick = torch.cat([torch.tensor([0, 1, 127, 128, n - 1, 32767, 32768, 32895, 32896], device="cuda"), torch.randint(0, n, (40,), generator=gen, device="cuda")])
    heads = [sampled({x: (y if x in "kv" else y[:, h:h + 1]) for x, y in t.items()}, pick, pick, D ** -0.5, 100, mq, mk) for h in range(G)]
    for h in range(G):
        plain.check({"dq": got["dq"][0, h][pick]}, {"dq": heads[h]["dq"]})
    # (of each head's part the sum, with the half step of each that is not there)
    plain.check({x: got[x][0, 0][pick] for x in ("dk", "dv")}, {x: tuple(sum(y[x][i] for y in heads) for i in range(2)) for x in ("dk", "dv")})


@pytest.mark.parametrize("n,D,K,G", [(33500, 64, 4, 2), (40000, 128, 8, 1), (9000, 128, 16, 8), (33000, 256, 4, 1)])
def test_assignments_of_long_sequences(n, D, K, G):
    """dg of some tokens in 64 bits: as rows over all columns, and as columns over all rows"""
    window, lam, scale = 64, 8.0, D ** -0.5
    t, gen = make(1, G, 1, n, D, 2)
    shape = fb.make_shape(G, 1, n, D, K, 1, window)
    g = torch.softmax(torch.randn((1, n, K), generator=gen, device="cuda"), -1)
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((1, G, n), device="cuda")
    fb.focus_gate_attn_fwd(shape, t["q"], t["k"], t["v"], g, lam, t["o"], t["lse"])
    got = run_bwd(shape, t, g=g, lam=lam)
    pick = torch.cat([torch.tensor([0, 63, 128, n - 1, min(n - 2, 32767), min(n - 3, 32768)], device="cuda"), torch.randint(0, n, (30,), generator=gen, device="cuda")])
    gd, at = g[0].double(), torch.arange(n, device="cuda")
    want = [torch.zeros((len(pick), K), dtype=torch.float64, device="cuda") for _ in range(2)]
    k, v = t["k"][0, 0].double(), t["v"][0, 0].double()
    for h in range(G):
        q, o, do, lse = (t[x][0, h].double() for x in ("q", "o", "do", "lse"))
        delta, base = (do * o).sum(-1), (do * o).abs().sum(-1)

        def part(i, j):
            """da and its bound (the terms of bwd_plain.backward)"""
            raw = scale * q[i] @ k[j].T
            d = at[i][:, None] - at[j][None]
            f = torch.where(d <= window, 1.0, torch.sigmoid(lam * gd[i] @ gd[j].T))
            p = torch.where(d >= 0, torch.exp(raw * f - lse[i][:, None]), 0.0)
            ds = p * (do[i] @ v[j].T - delta[i][:, None])
            es = p * (do[i].abs() @ v[j].abs().T + base[i][:, None]) * (plain.E + plain.E * (1 + (raw * f).abs()))
            s = torch.where(d <= window, 0.0, lam * f * (1 - f))
            return ds * raw * s, (es * raw.abs() + ds.abs() * plain.E * (1 + raw.abs())) * s + plain.E * (ds * raw * s).abs()
        a, e = part(pick, slice(0, n))
        b, c = part(slice(0, n), pick)
        for x, y, z in ((0, a, b), (1, e, c)):
            want[x] += y @ gd + z.T @ gd
    plain.check({"dg": got["dg"][0][pick][:, :K]}, {"dg": tuple(want)})


def test_several_launches_captured_and_on_two_streams():
    """(their sums lie in the workspace from launch to launch) the same bits from a graph replayed on new inputs, and from two calls at once"""
    n, D, G, K = 33500, 64, 3, 4
    shape = fb.make_shape(G, 1, n, D, K, 1, 50)
    cases = []
    for seed in (1, 2):
        t, gen = make(1, G, 1, n, D, seed)
        g = torch.softmax(torch.randn((1, n, K), generator=gen, device="cuda"), -1)
        t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((1, G, n), device="cuda")
        fb.focus_gate_attn_fwd(shape, t["q"], t["k"], t["v"], g, 6.0, t["o"], t["lse"])
        cases.append((t, g, run_bwd(shape, t, g=g, lam=6.0), run_bwd(shape, t)))
    size = (fb.focus_gate_attn_bwd_workspace_bytes(shape), fb.focus_attn_bwd_workspace_bytes(shape))
    spaces = [[torch.empty(x, dtype=torch.uint8, device="cuda").fill_(0xff) for x in size] for _ in cases]
    outs = [[{x: torch.empty_like(y) for x, y in r.items()} for r in c[2:]] for c in cases]

    def both(t, g, ws, out, stream=None):
        fb.focus_gate_attn_bwd(shape, t["q"], t["k"], t["v"], g, 6.0, t["o"], t["lse"], t["do"], *out[0].values(), ws[0], None, stream)
        fb.focus_attn_bwd(shape, t["q"], t["k"], t["v"], None, None, None, 0, t["o"], t["lse"], t["do"], *out[1].values(), ws[1], None, stream)

    same = lambda out, c: all(torch.equal(o[x], r[x]) for o, r in zip(out, c[2:]) for x in r)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(2):
        for c, ws, out, st in zip(cases, spaces, outs, streams):
            both(c[0], c[1], ws, out, st)
    torch.cuda.synchronize()
    assert same(outs[0], cases[0]) and same(outs[1], cases[1])
    t, g = {x: y.clone() for x, y in cases[0][0].items()}, cases[0][1].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(t, g, spaces[0], outs[0])
    for x in t:
        t[x].copy_(cases[1][0][x])
    g.copy_(cases[1][1])
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert same(outs[0], cases[1])
