"""The backward entry points as they are called: through csrc/marshal.cpp and through ctypes, with the same results and errors; on long and on many
sequences, and on tensors whose offsets pass 32 bits."""
import math

import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb
from test_gpu_attn_bwd import groups, make, run_bwd, tiles_of

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    pass


class Calls:
    """in the place of the module: counts how often it was asked and how often it answered; without `behind` it never does"""
    def __init__(self, behind=None):
        self.asked = self.answered = 0
        self.behind = behind

    def __getattr__(self, name):
        def call(*args):
            self.asked += 1
            rc = getattr(self.behind, name)(*args) if self.behind else None
            self.answered += rc is not None
            return rc
        return call


def everything(wrap, stream=None):
    B, Hq, Hkv, n, D, K, d, dg = 2, 4, 2, 150, 64, 4, 72, 5
    t, gen = make(B, Hq, Hkv, n, D, 1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    shape = fb.make_shape(Hq, Hkv, n, D, K, 2, 9, batch=B)
    mq, mk = groups(gen, B, Hq, n, K, 2), groups(gen, B, Hkv, n, K, 2)
    tiles = tiles_of(shape, mq, mk)
    g = torch.softmax(rnd(B, n, K), -1)
    o, lse, do = t["q"] * 0.5, rnd(B, Hq, n).abs() + 9, t["do"]
    h, Wg, C, ds = rnd(B, n, d).to(torch.bfloat16), rnd(d, dg), rnd(K, dg), rnd(B, n, K)
    new = torch.zeros_like
    out = [new(t["q"]), new(t["k"]), new(t["v"])]
    gout = [new(x) for x in out] + [new(g)]
    rout = [new(h), new(Wg), new(C)]
    status, norm = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    byte = lambda size: torch.zeros(size, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    fb.focus_attn_bwd(shape, wrap(t["q"]), t["k"], t["v"], mq, mk, tiles, 0, o, lse, do, *out, byte(fb.focus_attn_bwd_workspace_bytes(shape)), status, stream)
    fb.focus_gate_attn_bwd(shape, t["q"], wrap(t["k"]), t["v"], g, 3.0, o, lse, do, *gout, byte(fb.focus_gate_attn_bwd_workspace_bytes(shape)), status, stream)
    fb.focus_router_scores_bwd(shape, wrap(h), Wg, C, ds, *rout, byte(fb.focus_router_scores_bwd_workspace_bytes(shape, d, dg)), stream)
    fb.focus_grad_clip(fb.make_grad_list([rout[1], rout[2]]), 1.0, wrap(norm), byte(fb.focus_grad_clip_workspace_bytes()), stream)
    torch.cuda.synchronize()
    assert status[0].item() == 0
    return out + gout + rout + [norm]


def test_same_results_both_ways(monkeypatch):
    fb.lib()
    module = fb._marshal
    same = lambda t: t
    want = everything(same)
    side = torch.cuda.Stream()
    for wrap, stream, behind in ((same, None, module), (same, side, module), (lambda t: t.as_subclass(Sub), None, module), (same, None, None), (same, side, None)):
        calls = Calls(behind)
        monkeypatch.setattr(fb, "_marshal", calls)
        got = everything(wrap, stream)
        monkeypatch.setattr(fb, "_marshal", module)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert calls.asked == 5                                  # the tiles and the four
        if wrap is same and stream is None:
            assert calls.answered == (5 if behind else 0)


@pytest.mark.parametrize("direct", [True, False])
def test_same_errors_both_ways(monkeypatch, direct):
    fb.lib()
    if not direct:
        monkeypatch.setattr(fb, "_marshal", Calls())
    B, Hq, Hkv, n, D, K = 1, 2, 1, 40, 64, 4
    t, gen = make(B, Hq, Hkv, n, D, 1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, 9, batch=B)
    lse, g = torch.zeros((B, Hq, n), device="cuda"), torch.zeros((B, n, K), device="cuda")
    ws = torch.zeros(fb.focus_gate_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    new = torch.empty_like
    hard = dict(q=t["q"], k=t["k"], v=t["v"], mq=None, mk=None, tiles=None, layout=0, o=new(t["q"]), lse=lse, do=t["do"], dq=new(t["q"]), dk=new(t["k"]), dv=new(t["v"]), ws=ws)
    gate = dict(q=t["q"], k=t["k"], v=t["v"], g=g, lam=1.0, o=hard["o"], lse=lse, do=t["do"], dq=hard["dq"], dk=hard["dk"], dv=hard["dv"], dg=new(g), ws=ws)
    bad = [("q", t["q"].float()), ("dk", t["q"]), ("lse", lse.double()), ("lse", lse[..., :5]), ("o", hard["o"].cpu())]
    for call, args, more in ((fb.focus_attn_bwd, hard, [("mq", g)]), (fb.focus_gate_attn_bwd, gate, [("g", g[..., :2]), ("dg", g.double())])):
        for name, x in bad + more:
            with pytest.raises(AssertionError):
                call(shape, *dict(args, **{name: x}).values())
        with pytest.raises(fb.FocusError):
            call(shape, *dict(args, ws=ws[:64]).values())
        with pytest.raises(fb.FocusError):
            call(shape, *dict(args, dq=t["q"]).values())
    h, Wg, C, ds = torch.zeros((n, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((64, 4), device="cuda"), torch.zeros((K, 4), device="cuda"), torch.zeros((1, n, K), device="cuda")
    wr = torch.zeros(fb.focus_router_scores_bwd_workspace_bytes(shape, 64, 4), dtype=torch.uint8, device="cuda")
    router = dict(h=h, Wg=Wg, C=C, ds=ds, dh=new(h), dWg=new(Wg), dC=new(C), ws=wr)
    for name, x in (("h", h.float()), ("h", h[:7]), ("Wg", Wg.t()), ("ds", ds[0, :3]), ("dh", new(h)[:, :32]), ("dC", C.double())):
        with pytest.raises(AssertionError):
            fb.focus_router_scores_bwd(shape, *dict(router, **{name: x}).values())
    with pytest.raises(fb.FocusError):
        fb.focus_router_scores_bwd(shape, *dict(router, ws=wr[:16]).values())
    for grads, out in (([h.cpu()], None), ([Wg.t()], None), ([Wg.double()], None), ([Wg], [C]), ([Wg], [Wg.to(torch.bfloat16)])):
        with pytest.raises(AssertionError):
            fb.make_grad_list(grads, out)
    with pytest.raises(fb.FocusError):
        fb.focus_grad_clip(fb.make_grad_list([Wg]), -1.0, None, ws)
    with pytest.raises(AssertionError):
        fb.focus_grad_clip(fb.make_grad_list([Wg]), 1.0, lse, ws)


def forward(shape, t, mq=None, mk=None, tiles=None):
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty(t["q"].shape[:3], device="cuda")
    fb.focus_attn_fwd(shape, t["q"], t["k"], t["v"], mq, mk, tiles, 0, t["o"], t["lse"])


def sampled(t, rows, cols, scale, window=None, mq=None, mk=None):
    """dq of some rows and dk, dv of some columns of one head, in 64 bits, each with its bound (the terms of bwd_plain.backward)"""
    q, k, v, o, do, lse = (t[x][0, 0].double() for x in ("q", "k", "v", "o", "do", "lse"))
    n = q.shape[0]
    delta, base = (do * o).sum(-1), (do * o).abs().sum(-1)
    at = torch.arange(n, device="cuda")

    def part(i, j):
        x = scale * q[i] @ k[j].T
        keep = at[j][None] <= at[i][:, None]
        if mq is not None:
            keep &= (at[i][:, None] - at[j][None] <= window) | ((mq[0, 0][i][:, None] & mk[0, 0][j][None]) != 0)
        p = torch.where(keep, torch.exp(x - lse[i][:, None]), 0.0)
        ep = plain.E * (1 + x.abs())
        ds = p * (do[i] @ v[j].T - delta[i][:, None])
        es = p * (do[i].abs() @ v[j].abs().T + base[i][:, None]) * (plain.E + ep)
        return p, ds, plain.U * ds.abs() + es, p * (plain.U + ep)
    all_ = slice(0, n)
    _, ds, ws, _ = part(rows, all_)
    dq = scale * ds @ k
    out = {"dq": (dq, scale * ws @ k.abs() + plain.U * dq.abs())}
    p, ds, ws, wp = part(all_, cols)
    dk, dv = scale * ds.T @ q, p.T @ do
    out["dk"], out["dv"] = (dk, scale * ws.T @ q.abs() + plain.U * dk.abs()), (dv, wp.T @ do.abs() + plain.U * dv.abs())
    return out


@pytest.mark.parametrize("n,D,masks", [(40000, 64, True), (33001, 128, False), (9001, 256, True)])
def test_long_sequences(n, D, masks):
    """more than 256 tiles (a word of live tiles is 32), sums over tens of thousands of rows"""
    t, gen = make(1, 1, 1, n, D, 1)
    shape = fb.make_shape(1, 1, n, D, 8, 1, 500)
    mq, mk = (groups(gen, 1, 1, n, 8, 1) for _ in range(2)) if masks else (None, None)
    tiles = tiles_of(shape, mq, mk) if masks else None
    forward(shape, t, mq, mk, tiles)
    got = run_bwd(shape, t, mq, mk, tiles)
    pick = torch.cat([torch.tensor([0, 1, 127, 128, n - 1], device="cuda"), torch.randint(0, n, (40,), generator=gen, device="cuda")])
    want = sampled(t, pick, pick, D ** -0.5, 500, mq, mk)
    plain.check({x: got[x][0, 0][pick] for x in want}, want)


def test_many_short_sequences():
    B, Hq, Hkv, n, D, K, window, lam = 150, 6, 2, 37, 64, 4, 3, 8.0
    t, gen = make(B, Hq, Hkv, n, D, 2)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, batch=B)
    g = torch.softmax(torch.randn((B, n, K), generator=gen, device="cuda"), -1)
    for how in (dict(), dict(g=g.double(), lam=lam)):
        o, lse = plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window if how else n, **how)
        t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
        got = run_bwd(shape, t, g=g, lam=lam) if how else run_bwd(shape, t)
        plain.check(got, plain.backward(*(t[x] for x in ("q", "k", "v", "o", "lse", "do")), D ** -0.5, window if how else n, **how))


@pytest.mark.parametrize("gate", [False, True])
def test_offsets_beyond_32_bits(gate):
    """every tensor a piece of one of 300000 numbers a token, 5.4 GB: the same bits as from tensors side by side"""
    n, D, wide = 9000, 64, 300000
    t, gen = make(1, 2, 1, n, D, 3, token_major=False)
    shape = fb.make_shape(2, 1, n, D, 4, 1, 64)
    forward(shape, t)
    g = torch.softmax(torch.randn((1, n, 4), generator=gen, device="cuda"), -1) if gate else None
    want = run_bwd(shape, t, g=g, lam=5.0)
    big = torch.empty((1, 1, n, wide), dtype=torch.bfloat16, device="cuda")
    far, at = {}, 0
    for x in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
        H = 1 if x[-1] in "kv" else 2
        far[x] = big[..., at:at + H * D].view(1, n, H, D).transpose(1, 2)
        at += 2 * D + 37000
        if x in t:
            far[x].copy_(t[x])
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    args = [far[x] for x in ("q", "k", "v")]
    if gate:
        ws, dg = torch.empty(fb.focus_gate_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda"), torch.empty_like(g)
        fb.focus_gate_attn_bwd(shape, *args, g, 5.0, far["o"], t["lse"], far["do"], far["dq"], far["dk"], far["dv"], dg, ws, status)
        assert torch.equal(dg, want["dg"])
    else:
        ws = torch.empty(fb.focus_attn_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
        fb.focus_attn_bwd(shape, *args, None, None, None, 0, far["o"], t["lse"], far["do"], far["dq"], far["dk"], far["dv"], ws, status)
    assert status[0].item() == 0 and all(torch.equal(far[x], want[x]) for x in ("dq", "dk", "dv"))


def test_router_offsets_beyond_32_bits():
    n, d, wide = 9000, 136, 300000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    shape = fb.make_shape(1, 1, n, 64, 5, 1, 0)
    big = torch.empty((1, n, wide), dtype=torch.bfloat16, device="cuda")
    h, dh = big[..., 8:8 + d], big[..., 200000:200000 + d]
    h.copy_(torch.randn((1, n, d), generator=gen, device="cuda"))
    Wg, C, ds = (torch.randn(s, generator=gen, device="cuda") for s in ((d, 7), (5, 7), (1, n, 8)))
    out = []
    for x, y in ((h, dh), (h.contiguous(), torch.empty((1, n, d), dtype=torch.bfloat16, device="cuda"))):
        dWg, dC = torch.empty_like(Wg), torch.empty_like(C)
        ws = torch.empty(fb.focus_router_scores_bwd_workspace_bytes(shape, d, 7), dtype=torch.uint8, device="cuda")
        fb.focus_router_scores_bwd(shape, x, Wg, C, ds, y, dWg, dC, ws)
        out.append((y, dWg, dC))
    assert all(torch.equal(a, b) for a, b in zip(*out))
