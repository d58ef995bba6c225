"""focus_gate_attn_fwd and focus_gate_attn_bwd after one another on scores of some dozens, against 64-bit autograd of the whole formula, with its own o and
lse: the two calls take the gate's factor in different ways (the forward from the hardware's tanh)."""
import math

import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb
from test_gpu_attn_bwd import make, run_bwd

pytestmark = pytest.mark.gpu

GATE = 2.0 ** -12       # error of the forward's factor: half of what the hardware's tanh is off, 2^-11 of itself


@pytest.mark.parametrize("Hq,Hkv,n,D,K,window,lam,scale", [(4, 2, 300, 64, 4, 20, 10.0, 1.0), (2, 1, 260, 128, 8, 0, 5.0, 0.6), (2, 2, 200, 256, 4, 50, 10.0, 0.5), (2, 1, 400, 64, 16, 30, -6.0, 1.0),
                                                            (2, 1, 300, 128, 32, 5, 0.0, 0.5), (2, 2, 300, 64, 4, 16, -10.0, 0.3)])
def test_forward_and_backward(Hq, Hkv, n, D, K, window, lam, scale):
    t, gen = make(1, Hq, Hkv, n, D, n + D)
    g = torch.zeros((1, n, fb.focus_soft_ld(K)), device="cuda")
    g[..., :K] = torch.softmax(2 * torch.randn((1, n, K), generator=gen, device="cuda"), -1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, window, scale)
    t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty((1, Hq, n), device="cuda")
    fb.focus_gate_attn_fwd(shape, t["q"], t["k"], t["v"], g, lam, t["o"], t["lse"])
    got = run_bwd(shape, t, g=g, lam=lam)

    G = Hq // Hkv
    leaves = [t[x].double().requires_grad_() for x in "qkv"] + [g.double().requires_grad_()]
    o, _ = plain.forward(*leaves[:3], scale, window, g=leaves[3], lam=lam)
    want = dict(zip(("dq", "dk", "dv", "dg"), torch.autograd.grad(o, leaves, t["do"].double())))

    # the bounds: as in bwd_plain.backward, and besides the factor's error in p (its own, and by way of lse that of the row's others), and o as the forward
    # pass leaves it in delta: its probabilities off by as much and rounded to bf16, its result rounded
    q, do = t["q"].double(), t["do"].double()
    kr, vr = (t[x].double().repeat_interleave(G, 1) for x in "kv")
    gd, o = g.double(), o.detach()
    raw, x, slope, seen = plain.logits(q, kr, scale, window, gd, lam)
    x = x.masked_fill(~seen, -math.inf)
    p = torch.softmax(x, -1)
    size_x = raw.abs().masked_fill(~seen, 0.0)
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")
    far = (i - j > window).double()
    ep = plain.E * (1 + size_x) + GATE * size_x * far
    ep = ep + (p * ep).sum(-1, keepdim=True)
    size = do.abs() @ vr.abs().transpose(-1, -2) + (do * o).abs().sum(-1, keepdim=True)
    off = (do.abs() * (plain.U * o.abs() + (p * (ep + plain.U)) @ vr.abs())).sum(-1, keepdim=True)
    ds = p * (do @ vr.transpose(-1, -2) - (do * o).sum(-1, keepdim=True))
    es = p * (size * (plain.E + ep) + off * (1 + ep))
    T, fold = (lambda y: y.transpose(-1, -2)), (lambda y: y.unflatten(1, (Hkv, G)).sum(2))
    w = plain.U * (ds * slope).abs() + es * slope
    da = ds * raw * (slope_da := far * lam * slope * (1 - slope))
    ea = ((es * raw.abs() + ds.abs() * plain.E * (1 + raw.abs())) * slope_da.abs() + plain.E * da.abs()).sum(1)
    bound = {"dv": fold(T(p * (plain.U + ep)) @ do.abs()), "dq": scale * w @ kr.abs(), "dk": fold(scale * T(w) @ q.abs()), "dg": ea @ gd.abs() + T(ea) @ gd.abs()}
    want["dg"][..., K:] = 0
    plain.check(got, {y: (want[y], bound[y] + (plain.U if y != "dg" else 0.0) * want[y].abs()) for y in bound})
    # (the bounds are not so wide that anything would pass: on average the error is below a twentieth of the gradient's size)
    for y in want:
        if want[y].norm() > 0:
            assert (got[y].double() - want[y]).norm() <= 0.05 * want[y].norm(), (y, ((got[y].double() - want[y]).norm() / want[y].norm()).item())
