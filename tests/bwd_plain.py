"""Plain forms in 64 bits of the attention forward pass and its derivative, with the bounds that roundings give the derivative.

U is half a step of bf16 relative to the value (2^-8), E what fp32 arithmetic adds: sums of up to some thousand products and an
exponential whose argument is a few dozen, 2^-17 of the sum of the absolute terms covers both (a sum of N terms in fp32 is off by at most
N 2^-24 of that in any order, N <= 128 within a tile's product, and what tiles add lies behind it by the running sums' own half steps)."""
import math

import torch

U = 2.0 ** -8
E = 2.0 ** -17


def shared(mq, mk, G):
    """[B, Hq, n, n]: the two tokens have a group in common"""
    return (mq[..., :, None] & mk.repeat_interleave(G, 1)[..., None, :]) != 0


def logits(q, k, scale, window, g=None, lam=0.0, softcap=0.0, keep=None):
    """(raw, logit, d logit / d raw, kept) of every pair; q, k float64 [B, Hq, n, D] (k repeated for its query heads)"""
    n = q.shape[2]
    i, j = torch.arange(n, device=q.device)[:, None], torch.arange(n, device=q.device)
    raw = scale * q @ k.transpose(-1, -2)
    seen, near = (j <= i).expand(raw.shape), i - j <= window
    if keep is not None:
        seen = seen & (near | keep)
    slope = torch.ones_like(raw)
    logit = raw
    if g is not None:
        slope = torch.where(near, 1.0, torch.sigmoid(lam * g @ g.transpose(-1, -2))[:, None]).expand(raw.shape)
        logit = raw * slope
    elif softcap:
        t = torch.tanh(raw / softcap)
        logit, slope = softcap * t, 1 - t * t
    return raw, logit, slope, seen


def forward(q, k, v, scale, window, **how):
    """o, lse in 64 bits"""
    G = q.shape[1] // k.shape[1]
    q, k, v = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    _, x, _, seen = logits(q, k, scale, window, **how)
    x = x.masked_fill(~seen, -math.inf)
    return torch.softmax(x, -1) @ v, torch.logsumexp(x, -1)


def backward(q, k, v, o, lse, do, scale, window, g=None, lam=0.0, softcap=0.0, keep=None):
    """{name: (value, bound on the kernel's error)}; o and lse are those the kernel is given"""
    B, Hq, n, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    q, o, do, lse = q.double(), o.double(), do.double(), lse.double()
    kr, vr = k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    g = None if g is None else g.double()
    raw, x, slope, seen = logits(q, kr, scale, window, g, lam, softcap, keep)
    p = torch.where(seen, torch.exp(x - lse[..., None]), 0.0).nan_to_num(posinf=0.0)
    dp = do @ vr.transpose(-1, -2)
    size = do.abs() @ vr.abs().transpose(-1, -2) + (do * o).abs().sum(-1, keepdim=True)      # of what ds is a difference of
    ds = p * (dp - (do * o).sum(-1, keepdim=True))
    # relative errors of p: the argument's (and the hardware tanh's, 2^-10.98 of the capped logit), of the slope 1 - t^2: twice t^2 that
    ep = E * (1 + x.abs())
    if softcap:
        ep = ep + 2.0 ** -10.98 * x.abs()
    fold = lambda t: t.unflatten(1, (Hkv, G)).sum(2)
    T = lambda t: t.transpose(-1, -2)
    out = {}
    dv = fold(T(p) @ do)
    out["dv"] = (dv, fold(T(p * (U + ep)) @ do.abs()) + U * dv.abs())
    es = p * size * (E + ep)                               # ds in fp32
    dx = ds * slope
    ex = es * slope + (2 * 2.0 ** -10.98 * (x / softcap) ** 2 * ds.abs() if softcap else 0.0)
    for name, a, b, sel in (("dq", dx, kr, None), ("dk", T(dx), q, fold)):
        w = (U * dx.abs() + ex) if sel is None else T(U * dx.abs() + ex)
        val, err = scale * (a @ b), scale * (w @ b.abs())
        if sel is not None:
            val, err = sel(val), sel(err)
        out[name] = (val, err + U * val.abs())
    if g is not None:
        i, j = torch.arange(n, device=q.device)[:, None], torch.arange(n, device=q.device)
        slope_da = torch.where(i - j <= window, 0.0, lam * slope * (1 - slope))
        da, ea = (ds * raw * slope_da).sum(1), ((es * raw.abs() + ds.abs() * E * (1 + raw.abs())) * slope_da).sum(1)
        ea = ea + E * (ds * raw * slope_da).abs().sum(1)
        out["dg"] = (da @ g + T(da) @ g, ea @ g.abs() + T(ea) @ g.abs())
    return out


def check(got, want):
    for name, (val, bound) in want.items():
        err = (got[name].double() - val).abs()
        tiny = 1e-30
        worst = (err / (bound + tiny)).max().item()
        assert torch.isfinite(got[name]).all() and worst <= 1.0, (name, worst, err.max().item(), val.abs().max().item())
