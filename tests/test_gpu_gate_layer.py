"""The training step of a layer with soft groups: the calls after one another as GateLayer makes them, each on what the one before it left, against the
formulas in 64 bits, with the bounds carried along; and against differences of the loss."""
import math

import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200.gate_layer import GateLayer

pytestmark = pytest.mark.gpu

CASES = [  # B, Hq, Hkv, n, D, K, d_model, d_g, window, lambda
    (1, 2, 1, 90, 64, 4, 256, 16, 8, 6.0), (2, 4, 2, 65, 128, 3, 96, 5, 0, 10.0), (1, 1, 1, 1, 64, 2, 64, 4, 0, 5.0), (1, 2, 2, 70, 256, 8, 136, 33, 20, 0.0),
]
TAU, ITERS = 0.3, 6


def inputs(B, Hq, Hkv, n, D, K, d, dg, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    t = {x: rnd(B, n, H, D).to(torch.bfloat16).transpose(1, 2) for x, H in (("q", Hq), ("k", Hkv), ("v", Hkv), ("do", Hq))}
    t["h"] = rnd(B, n, d).to(torch.bfloat16)
    return t, rnd(d, dg) / d ** 0.5, 0.3 * rnd(K, dg), gen


def sinkhorn64(S, tau, iters):
    Q = torch.exp(S / tau)
    for _ in range(iters):
        Q = Q / Q.sum(1, keepdim=True)
        Q = Q / Q.sum(2, keepdim=True)
    return Q


def step(layer, t, Wg, C, stream=None):
    out = {x: torch.full_like(t[x[1:]], math.nan) for x in ("dq", "dk", "dv", "dh")}
    o = torch.full_like(t["q"], math.nan)
    layer.forward(t["h"], t["q"], t["k"], t["v"], Wg, C, o, stream)
    layer.backward(t["h"], t["q"], t["k"], t["v"], Wg, C, o, t["do"], out["dq"], out["dk"], out["dv"], out["dh"], stream)
    return o, out


def chain(layer, t, Wg, C, o, window, lam):
    """{name: (value, bound)} of the gradients behind the gate, from the scores, assignments, o and lse that the layer has"""
    K, scale = layer.shape.K, layer.shape.D ** -0.5
    want = plain.backward(t["q"], t["k"], t["v"], o, layer.lse, t["do"], scale, window, g=layer.g, lam=lam)
    dg, eg = (x[..., :K] for x in want.pop("dg"))
    S = layer.scores.double()[..., :K]
    jac = torch.autograd.functional.jacobian(lambda x: sinkhorn64(x, TAU, ITERS), S, vectorize=True).flatten(0, 2).flatten(1)
    ds, es = dg.flatten() @ jac, eg.flatten() @ jac.abs()
    es = es + 2e-4 * ds.abs().max()                       # focus_sinkhorn_bwd's own tolerance
    ds, es = ds.view_as(dg), es.view_as(dg)
    h, W, Cd = t["h"].double(), Wg.double(), C.double()
    hs, ts = torch.einsum("bng,bnd->gd", ds, h), torch.einsum("bng,bnd->gd", es + plain.E * ds.abs(), h.abs())
    want["dC"] = (hs @ W, ts @ W.abs() + plain.E * (hs.abs() @ W.abs()))
    want["dWg"] = (hs.T @ Cd, ts.T @ Cd.abs() + plain.E * (hs.abs().T @ Cd.abs()))
    F, Fa = Cd @ W.T, Cd.abs() @ W.abs().T
    dh = ds @ F
    # dS and F in two bf16 terms each: 2^-16 (a quarter of half a step squared each, twice that counted) and fp32 sums
    want["dh"] = (dh, es @ Fa + ds.abs() @ Fa * (plain.E + 2.0 ** -15) + plain.U * dh.abs())
    return want


@pytest.mark.parametrize("B,Hq,Hkv,n,D,K,d,dg,window,lam", CASES)
def test_step_and_clip(B, Hq, Hkv, n, D, K, d, dg, window, lam):
    t, Wg, C, _ = inputs(B, Hq, Hkv, n, D, K, d, dg, n + D)
    layer = GateLayer(B, Hq, Hkv, n, D, K, d, dg, window, lam, TAU, ITERS)
    o, out = step(layer, t, Wg, C)
    out = dict(out, dWg=layer.dWg, dC=layer.dC)
    torch.cuda.synchronize()
    assert layer.status.tolist()[0] == 0
    plain.check(out, chain(layer, t, Wg, C, o, window, lam))
    # the gradients of one step clipped together, fp32 and bf16: every square counts once, half a step for what is rounded
    grads = [out[x] for x in ("dWg", "dC", "dh")] + [out[x].contiguous() for x in ("dq", "dk", "dv")]
    before = [x.double() for x in grads]
    norm = math.sqrt(sum(x.square().sum().item() for x in before))
    layer.clip(fb.make_grad_list(grads), norm / 3)
    torch.cuda.synchronize()
    assert abs(layer.norm.item() - norm) <= 2.0 ** -22 * norm
    for x, y in zip(grads, before):
        eps = torch.finfo(x.dtype).eps / 2 + 2.0 ** -22
        assert ((x.double() - y / 3).abs() <= eps * y.abs() / 3 + 1e-38).all()


def test_against_differences_of_the_loss():
    """the loss sum(o do) of the whole chain in 64 bits, a step of 1e-3 either way in W_g, C and h, against the layer's gradients along it"""
    B, Hq, Hkv, n, D, K, d, dg, window, lam = CASES[0]
    t, Wg, C, gen = inputs(B, Hq, Hkv, n, D, K, d, dg, 3)
    layer = GateLayer(B, Hq, Hkv, n, D, K, d, dg, window, lam, TAU, ITERS)
    o, out = step(layer, t, Wg, C)
    got = dict(dWg=layer.dWg, dC=layer.dC, dh=out["dh"])
    want = chain(layer, t, Wg, C, o, window, lam)

    def loss(h, W, Cd):
        g = sinkhorn64(h @ W @ Cd.T, TAU, ITERS)
        return (plain.forward(t["q"], t["k"], t["v"], D ** -0.5, window, g=g, lam=lam)[0] * t["do"].double()).sum()

    # o's rounding moves delta, and with it every ds, by at most half a step of sum |o do|: carried along like an error of dg
    at = {"h": t["h"].double(), "Wg": Wg.double(), "C": C.double()}
    leaf = {x: y.clone().requires_grad_() for x, y in at.items()}
    exact = dict(zip(leaf, torch.autograd.grad(loss(*leaf.values()), list(leaf.values()))))
    for x in ("Wg", "C", "h"):
        u = torch.randn(at[x].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = ({y: z + s * 1e-3 * u if y == x else z for y, z in at.items()} for s in (1, -1))
        slope = (loss(*up.values()) - loss(*down.values())) / 2e-3
        along = (exact[x] * u).sum()
        assert (slope - along).abs() <= 1e-2 * along.abs() + 1e-3 * exact[x].norm()              # (the cubic term of the step: the formula itself)
        mine = (got["d" + x].double() * u).sum()
        bound = (want["d" + x][1] * u.abs()).sum() + ((want["d" + x][0] - exact[x]).abs() * u.abs()).sum()
        assert (mine - along).abs() <= bound and (want["d" + x][0] - exact[x]).norm() <= 2e-2 * exact[x].norm(), (x, mine.item(), along.item(), bound.item())


def test_captured_and_replayed_on_new_inputs_on_a_stream():
    B, Hq, Hkv, n, D, K, d, dg, window, lam = 1, 4, 2, 300, 128, 4, 512, 16, 30, 8.0
    t, Wg, C, _ = inputs(B, Hq, Hkv, n, D, K, d, dg, 1)
    u, Wu, Cu, _ = inputs(B, Hq, Hkv, n, D, K, d, dg, 2)
    other, layer = (GateLayer(B, Hq, Hkv, n, D, K, d, dg, window, lam, TAU, ITERS) for _ in range(2))
    _, want = step(other, u, Wu, Cu)
    grads = fb.make_grad_list([other.dWg, other.dC])
    other.clip(grads, 1e-3)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step(layer, t, Wg, C)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        _, out = step(layer, t, Wg, C)
        layer.clip(fb.make_grad_list([layer.dWg, layer.dC]), 1e-3)
    for x in t:
        t[x].copy_(u[x])
    Wg.copy_(Wu)
    C.copy_(Cu)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[x], want[x]) for x in want)
    assert torch.equal(layer.dWg, other.dWg) and torch.equal(layer.dC, other.dC) and torch.equal(layer.norm, other.norm) and layer.status.tolist()[0] == 0
