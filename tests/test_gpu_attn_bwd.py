"""focus_attn_bwd and focus_gate_attn_bwd against the formulas in 64 bits (bwd_plain.py), against differences of the forward pass, and as
they are used: strided, on other streams, captured, after the forward kernels."""
import math

import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb

pytestmark = pytest.mark.gpu


def make(B, Hq, Hkv, n, D, seed, token_major=True):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = {}
    for x, H in (("q", Hq), ("k", Hkv), ("v", Hkv), ("do", Hq)):
        shape = (B, n, H, D) if token_major else (B, H, n, D)
        t[x] = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
        if token_major:
            t[x] = t[x].transpose(1, 2)
    return t, gen


def groups(gen, B, H, n, K, topk):
    pick = torch.rand((B, H, n, K), generator=gen, device="cuda").argsort(-1) < topk
    return (pick.int() << torch.arange(K, device="cuda", dtype=torch.int32)).sum(-1).to(torch.int32)


def run_bwd(shape, t, mq=None, mk=None, tiles=None, layout=0, g=None, lam=0.0, status=None, stream=None):
    out = {"dq": torch.full_like(t["q"], math.nan), "dk": torch.full_like(t["k"], math.nan), "dv": torch.full_like(t["v"], math.nan)}
    status = torch.zeros(4, dtype=torch.int32, device="cuda") if status is None else status
    if g is None:
        ws = torch.empty(fb.focus_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda").fill_(0xff)
        fb.focus_attn_bwd(shape, t["q"], t["k"], t["v"], mq, mk, tiles, layout, t["o"], t["lse"], t["do"], out["dq"], out["dk"], out["dv"], ws, status, stream)
    else:
        out["dg"] = torch.full_like(g, math.nan)
        ws = torch.empty(fb.focus_gate_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda").fill_(0xff)
        fb.focus_gate_attn_bwd(shape, t["q"], t["k"], t["v"], g, lam, t["o"], t["lse"], t["do"], out["dq"], out["dk"], out["dv"], out["dg"], ws, status, stream)
    torch.cuda.synchronize()
    assert status.tolist()[0] == 0, status.tolist()
    return out


def tiles_of(shape, mq, mk, layout=0):
    ws = fb.alloc_workspace(shape, layout)
    fb.focus_build_tiles(shape, mq, mk, layout, ws)
    return ws


HARD = [  # B, Hq, Hkv, n, D, K, topk, window, softcap
    (1, 1, 1, 1, 64, 4, 2, 0, 0.0), (2, 2, 1, 2, 128, 4, 1, 0, 0.0), (1, 4, 2, 63, 64, 4, 2, 5, 0.0), (1, 2, 2, 64, 128, 8, 1, 16, 0.0),
    (1, 3, 1, 65, 64, 4, 1, 0, 0.0), (2, 2, 1, 127, 128, 1, 1, 3, 0.0), (1, 2, 1, 128, 128, 4, 2, 127, 0.0), (1, 2, 1, 129, 64, 32, 3, 7, 0.0),
    (1, 4, 1, 200, 128, 4, 1, 1000, 0.0), (2, 6, 2, 257, 64, 16, 2, 64, 0.0), (1, 4, 2, 500, 128, 4, 2, 64, 0.0), (1, 2, 1, 1000, 128, 8, 1, 33, 0.0),
    (1, 2, 1, 385, 256, 4, 1, 40, 50.0), (1, 2, 2, 130, 256, 4, 2, 300, 0.0), (2, 2, 1, 300, 64, 4, 1, 20, 30.0), (1, 2, 1, 257, 128, 4, 1, 20, 5.0),
    (1, 1, 1, 2100, 64, 8, 1, 100, 0.0), (3, 8, 8, 140, 64, 4, 2, 9, 0.0), (1, 16, 1, 150, 128, 4, 1, 30, 0.0), (1, 4, 4, 700, 256, 4, 2, 100, 0.0),
]


@pytest.mark.parametrize("B,Hq,Hkv,n,D,K,topk,window,softcap", HARD)
def test_hard_mask(B, Hq, Hkv, n, D, K, topk, window, softcap):
    t, gen = make(B, Hq, Hkv, n, D, n + D)
    mq, mk = groups(gen, B, Hq, n, K, topk), groups(gen, B, Hkv, n, K, topk)
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, window, 0.0, softcap, batch=B)
    how = dict(softcap=softcap, keep=plain.shared(mq, mk, Hq // Hkv))
    o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, **how)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    got = run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk))
    plain.check(got, plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, **how))


@pytest.mark.parametrize("B,Hq,Hkv,n,D,scale,softcap", [(1, 1, 1, 1, 64, 0.0, 0.0), (1, 2, 1, 129, 128, 0.3, 0.0), (3, 4, 2, 333, 64, 0.0, 0.0), (1, 2, 1, 640, 128, 0.0, 20.0),
                                                        (2, 2, 2, 256, 256, 0.05, 0.0), (1, 8, 2, 511, 128, 0.0, 0.0), (1, 5, 1, 190, 256, 0.0, 10.0)])
def test_every_causal_pair(B, Hq, Hkv, n, D, scale, softcap):
    t, _ = make(B, Hq, Hkv, n, D, n, token_major=False)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 1, 3, scale, softcap, batch=B)
    sc = scale or D ** -0.5
    o, lse = plain.forward(t["q"], t["k"], t["v"], sc, n, softcap=softcap)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    plain.check(run_bwd(shape, t), plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), sc, n, softcap=softcap))


GATE = [  # B, Hq, Hkv, n, D, K, window, lambda
    (1, 1, 1, 1, 64, 4, 0, 10.0), (2, 2, 1, 2, 128, 3, 0, 5.0), (1, 4, 2, 130, 64, 4, 0, 10.0), (2, 2, 1, 257, 128, 8, 64, 10.0), (1, 3, 1, 200, 64, 7, 16, 30.0),
    (1, 2, 2, 300, 128, 16, 10, 10.0), (1, 2, 1, 260, 64, 32, 5, 10.0), (1, 2, 1, 140, 128, 32, 0, 8.0), (1, 2, 1, 270, 256, 8, 30, 10.0), (1, 2, 1, 150, 256, 16, 0, -4.0),
    (1, 4, 4, 500, 64, 1, 100, 10.0), (1, 2, 1, 400, 128, 4, 1000, 10.0), (1, 4, 1, 900, 128, 4, 64, 10.0),
]


@pytest.mark.parametrize("B,Hq,Hkv,n,D,K,window,lam", GATE)
def test_gate(B, Hq, Hkv, n, D, K, window, lam):
    t, gen = make(B, Hq, Hkv, n, D, n + K)
    g = torch.zeros((B, n, fb.focus_soft_ld(K)), device="cuda")
    g[..., :K] = torch.softmax(2 * torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, batch=B)
    o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, g=g.double(), lam=lam)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    got = run_bwd(shape, t, g=g, lam=lam)
    want = plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, g=g, lam=lam)
    want["dg"][0][..., K:] = 0
    plain.check(got, want)
    assert (got["dg"][..., K:] == 0).all()


def test_against_differences_of_the_forward_pass():
    """the loss sum(o do) a step of 1e-3 along a random direction either way, in 64 bits, against the gradients times that direction"""
    B, Hq, Hkv, n, D, K, window, lam = 1, 2, 1, 200, 64, 4, 20, 6.0
    t, gen = make(B, Hq, Hkv, n, D, 5)
    g = torch.softmax(torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    mq, mk = groups(gen, B, Hq, n, K, 1), groups(gen, B, Hkv, n, K, 1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, batch=B)
    for how in (dict(keep=plain.shared(mq, mk, Hq // Hkv)), dict(g=g.double(), lam=lam)):
        o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, **how)
        t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
        got = run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk)) if "keep" in how else run_bwd(shape, t, g=g, lam=lam)
        want = plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, **how)
        for x in ("q", "k", "v") + (("g",) if "g" in how else ()):
            base = how["g"] if x == "g" else t[x].double()
            u = torch.randn(base.shape, generator=gen, device="cuda", dtype=torch.float64)
            loss = []
            for sign in (1, -1):
                moved = {y: t[y].double() for y in ("q", "k", "v")}
                h = dict(how)
                (h if x == "g" else moved)[x] = base + sign * 1e-3 * u
                loss.append((plain.forward(moved["q"], moved["k"], moved["v"], D ** -0.5, window, **h)[0] * t["do"].double()).sum())
            slope = (loss[0] - loss[1]) / 2e-3
            mine = (got["d" + x].double() * u).sum()
            # the gradient's own bound along u, o's rounding (half a step of each number of o times do in every delta), and the cubic term of the step
            do, op = t["do"].double(), t["o"].double()
            bound = (want["d" + x][1] * u.abs()).sum() + plain.U * (want["d" + x][0] * u).abs().sum() + 1e-2 * slope.abs()
            assert (mine - slope).abs() <= bound, (x, mine.item(), slope.item(), bound.item())


@pytest.mark.parametrize("layout", [1, 3, 4])
def test_workspaces_of_the_sorted_layouts(layout):
    B, Hq, Hkv, n, D, K, topk, window = 1, 4, 2, 700, 128, 4, 2, 50
    t, gen = make(B, Hq, Hkv, n, D, 3)
    mq, mk = groups(gen, B, Hq, n, K, topk), groups(gen, B, Hkv, n, K, topk)
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, window, batch=B)
    o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, keep=plain.shared(mq, mk, 2))
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    a, b = run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk)), run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk, layout), layout)
    assert all(torch.equal(a[x], b[x]) for x in a)


def test_runs_of_groups_leave_tiles_out():
    """stretches of 300 tokens with one group each: most pairs of tiles hold no pair"""
    B, Hq, Hkv, n, D, K, window = 1, 4, 2, 2500, 64, 8, 100
    t, gen = make(B, Hq, Hkv, n, D, 9)
    m = (1 << torch.randint(0, K, (n // 300 + 1,), generator=gen, device="cuda")).to(torch.int32).repeat_interleave(300)[:n]
    mq, mk = m.expand(B, Hq, n).contiguous(), m.expand(B, Hkv, n).contiguous()
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, batch=B)
    how = dict(keep=plain.shared(mq, mk, 2))
    o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, **how)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    plain.check(run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk)), plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, **how))


def dense_case(seed=1, B=1, Hq=4, Hkv=2, n=600, D=128):
    t, _ = make(B, Hq, Hkv, n, D, seed)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 1, 3, batch=B)
    o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, n)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    return shape, t


def test_same_bits_every_time_and_on_two_streams_at_once():
    (s1, t1), (s2, t2) = dense_case(1), dense_case(2, n=900)
    a1, a2 = run_bwd(s1, t1), run_bwd(s2, t2)
    outs = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, t, st in ((s1, t1, streams[0]), (s2, t2, streams[1])):
        out = [torch.empty_like(t[x]) for x in ("q", "k", "v")]
        ws = torch.empty(fb.focus_attn_bwd_workspace_bytes(s), dtype=torch.uint8, device="cuda")
        st.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            fb.focus_attn_bwd(s, t["q"], t["k"], t["v"], None, None, None, 0, t["o"], t["lse"], t["do"], *out, ws, None, st)
        outs.append((out, ws))
    torch.cuda.synchronize()
    for a, (out, _) in ((a1, outs[0]), (a2, outs[1])):
        assert all(torch.equal(a[x], y) for x, y in zip(("dq", "dk", "dv"), out))


def test_captured_and_replayed_on_new_inputs():
    shape, t = dense_case(3)
    _, u = dense_case(4)
    g = torch.rand((1, 600, 4), device="cuda")
    out = [torch.empty_like(t[x]) for x in ("q", "k", "v")]
    gout = [torch.empty_like(t[x]) for x in ("q", "k", "v")] + [torch.empty_like(g)]
    ws = torch.empty(fb.focus_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    wsg = torch.empty(fb.focus_gate_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")

    def step():
        fb.focus_attn_bwd(shape, t["q"], t["k"], t["v"], None, None, None, 0, t["o"], t["lse"], t["do"], *out, ws)
        fb.focus_gate_attn_bwd(shape, t["q"], t["k"], t["v"], g, 4.0, t["o"], t["lse"], t["do"], *gout, wsg)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    want, wantg = run_bwd(shape, u), run_bwd(shape, u, g=g, lam=4.0)
    for x in t:
        t[x].copy_(u[x])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want.values())) and all(torch.equal(a, b) for a, b in zip(gout, wantg.values()))


def test_writes_its_own_rows_only():
    """outputs in the middle of larger buffers, n no multiple of a tile: what lies around stays"""
    shape, t = dense_case(6, n=150)
    big = {x: torch.full((1, H, 200, 160), 7.0, dtype=torch.bfloat16, device="cuda") for x, H in (("dq", 4), ("dk", 2), ("dv", 2))}
    view = {x: y[:, :, 20:170, 16:144] for x, y in big.items()}
    want = run_bwd(shape, t)
    ws = torch.empty(fb.focus_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    fb.focus_attn_bwd(shape, t["q"], t["k"], t["v"], None, None, None, 0, t["o"], t["lse"], t["do"], view["dq"], view["dk"], view["dv"], ws)
    torch.cuda.synchronize()
    for x in big:
        assert torch.equal(view[x], want[x])
        view[x].fill_(7.0)
        assert (big[x] == 7.0).all()


def test_rows_without_a_pair_have_no_gradient():
    """lse of -inf (a row that a partial pass left empty): its probabilities are 0"""
    shape, t = dense_case(7, n=260)
    t["lse"][:, :, 100:140] = -math.inf
    got = run_bwd(shape, t)
    want = plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), 128 ** -0.5, 260)
    plain.check(got, want)
    assert (got["dq"][:, :, 100:140] == 0).all()


def test_behind_the_forward_kernels():
    """assignments, tiles, forward pass and backward pass by the library alone, against the formula on what the forward pass left"""
    B, Hq, Hkv, n, D, K, topk, window = 2, 4, 2, 777, 128, 4, 2, 60
    t, gen = make(B, Hq, Hkv, n, D, 11)
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, window, batch=B)
    C = torch.randn((Hkv, K, D), generator=gen, device="cuda")
    mq, mk = torch.empty((B, Hq, n), dtype=torch.int32, device="cuda"), torch.empty((B, Hkv, n), dtype=torch.int32, device="cuda")
    fb.focus_assign(shape, t["q"], Hq, C, mq)
    fb.focus_assign(shape, t["k"], Hkv, C, mk)
    tiles = tiles_of(shape, mq, mk)
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((B, Hq, n), device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    fb.focus_attn_fwd(shape, t["q"], t["k"], t["v"], mq, mk, tiles, 0, t["o"], t["lse"], status)
    got = run_bwd(shape, t, mq, mk, tiles, status=status)
    plain.check(got, plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, keep=plain.shared(mq, mk, 2)))


@pytest.mark.parametrize("B,Hq,Hkv,n,D,K", [(1, 2, 1, 9000, 64, 4), (1, 2, 1, 5000, 64, 8), (1, 2, 1, 5000, 128, 4), (1, 2, 1, 3000, 128, 32), (1, 2, 1, 3000, 256, 8), (4, 12, 12, 1000, 64, 4)])
def test_gate_same_bits_every_time(B, Hq, Hkv, n, D, K):
    t, gen = make(B, Hq, Hkv, n, D, 3)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, 64, batch=B)
    g = torch.softmax(torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((B, Hq, n), device="cuda")
    fb.focus_gate_attn_fwd(shape, t["q"], t["k"], t["v"], g, 5.0, t["o"], t["lse"])
    first = run_bwd(shape, t, g=g, lam=5.0)
    for _ in range(8):
        again = run_bwd(shape, t, g=g, lam=5.0)
        assert all(torch.equal(first[x], again[x]) for x in first)


@pytest.mark.parametrize("B,Hq,Hkv,n,D,window", [(1, 8, 1, 700, 128, 30), (2, 6, 1, 600, 64, 9), (1, 12, 2, 515, 128, 1000), (1, 16, 2, 300, 256, 20)])
def test_query_heads_in_parts(B, Hq, Hkv, n, D, window):
    """so few KV heads that their query heads go to several blocks, six of them in parts of two or three too; outputs with strides of their own"""
    K, lam = 4, 7.0
    t, gen = make(B, Hq, Hkv, n, D, n)
    mq, mk = groups(gen, B, Hq, n, K, 1), groups(gen, B, Hkv, n, K, 1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, batch=B)
    g = torch.softmax(torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    for how in (dict(keep=plain.shared(mq, mk, Hq // Hkv)), dict(g=g.double(), lam=lam)):
        o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, **how)
        t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
        got = run_bwd(shape, t, mq, mk, tiles_of(shape, mq, mk)) if "keep" in how else run_bwd(shape, t, g=g, lam=lam)
        plain.check(got, plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window, **how))
