"""focus_attn_bwd with scores beyond their cap, where the cap's slope 1 - tanh^2 is small: it keeps its relative precision there."""
import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb
from test_gpu_attn_bwd import run_bwd

pytestmark = pytest.mark.gpu

TANH = 2.0 ** -10.98        # relative error of the hardware's tanh


def backward(q, k, v, o, lse, do, scale, cap):
    """{name: (value, bound)} as bwd_plain.backward, but for the slope: 4 e / (1 + e)^2, e = exp(-2 |raw / cap|), in 64 bits, and as its error
    that of e (fp32's argument and exponential: E of them), and of (1 + |t|)^2 with the hardware's t: at most twice TANH t / (1 + t), so TANH"""
    q, k, v, o, do, lse = (x.double() for x in (q, k, v, o, do, lse))
    n = q.shape[2]
    raw = scale * q @ k.transpose(-1, -2)
    t, e = torch.tanh(raw / cap), torch.exp(-2 * (raw / cap).abs())
    x, slope = cap * t, 4 * e / (1 + e) ** 2
    seen = torch.ones(n, n, dtype=torch.bool, device=q.device).tril()
    p = torch.where(seen, torch.exp(x - lse[..., None]), 0.0)
    delta = (do * o).sum(-1, keepdim=True)
    ds = p * (do @ v.transpose(-1, -2) - delta)
    size = p * (do.abs() @ v.abs().transpose(-1, -2) + (do * o).abs().sum(-1, keepdim=True))
    ep = plain.E * (1 + x.abs()) + TANH * x.abs()
    err = slope * (size * (plain.E + ep) + ds.abs() * (plain.U + TANH + plain.E * (1 + 2 * (raw / cap).abs())))
    dx, T = ds * slope, lambda y: y.transpose(-1, -2)
    out = {}
    for name, a, w, b in (("dq", dx, err, k), ("dk", T(dx), T(err), q)):
        val = scale * a @ b
        out[name] = (val, scale * w @ b.abs() + plain.U * val.abs())
    return out


@pytest.mark.parametrize("D,cap,lo,hi", [(64, 2.0, 4.0, 10.0), (128, 2.0, 6.0, 9.0), (256, 2.0, 4.0, 10.0), (128, 30.0, 5.0, 9.5), (256, 50.0, 0.0, 9.0), (64, 5.0, 0.0, 1.0), (128, 2.0, 0.0, 3.4), (64, 10.0, 3.2, 3.8), (128, 1.0, 15.0, 30.0)])
def test_scores_beyond_the_cap(D, cap, lo, hi):
    """the first dimension gives a row all of whose scores are some lo to hi caps, of either sign, the others what its gradient is made of"""
    n, scale = 150, 0.5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(D)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
    q, k, v, do = 0.02 * cap * rnd(1, 2, n, D), rnd(1, 1, n, D), rnd(1, 1, n, D), rnd(1, 2, n, D)
    level = torch.linspace(lo, hi, n, device="cuda")[torch.randperm(n, generator=gen, device="cuda")]
    q[..., 0] = cap / scale * level * rnd(1, 2, n).sign()
    k[..., 0] = 1
    t = {x: y.to(torch.bfloat16) for x, y in (("q", q), ("k", k), ("v", v), ("do", do))}
    o, lse = plain.forward(t["q"], t["k"], t["v"], scale, n, softcap=cap)
    t["o"], t["lse"] = o.to(torch.bfloat16), lse.float()
    got = run_bwd(fb.make_shape(2, 1, n, D, 4, 1, 0, scale, cap), t)
    # (dk of both query heads)
    fold = backward(t["q"], t["k"].expand(1, 2, n, D), t["v"].expand(1, 2, n, D), *(t[x] for x in ("o", "lse", "do")), scale, cap)
    fold["dk"] = tuple(x.sum(1, keepdim=True) for x in fold["dk"])
    plain.check(got, fold)
