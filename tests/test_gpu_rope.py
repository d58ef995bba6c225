"""focus_qk_norm_rope and its derivative against the formulas in 64 bits.

Tolerances: the result is rounded to bf16 once (half a step: 2^-8 of the value).  Before that, in fp32: the mean of squares is a sum of
at most 32 products a lane and five exchanges, all positive (2^-18 of it, half of that in the root), a handful of products (2^-24 each), and
sine and cosine of an angle reduced in 64 bits (2^-21 absolute, the angle's rounding to fp32 among it): 2^-17 of the larger of the pair, or of
the row's largest for the derivative, whose mean is a sum of products of either sign.  Weight gradients are fp32 sums of one term per row, in
chains of at most rows / 8 + 96: that many times 2^-24 of the sum of magnitudes, and 2^-18 of it for the terms themselves."""
import math

import pytest
import torch

from paper_2604_03260_b200 import binding as fb

pytestmark = pytest.mark.gpu


def turned(x, pos, freq, interleaved, rotary, amplitude, sign=1.0):
    """x [B, H, n, D] fp64, pos [B, n]"""
    z = pos.double()[:, None, :, None] * freq.double()
    c, s = amplitude * torch.cos(z), sign * amplitude * torch.sin(z)
    i = torch.arange(rotary // 2, device=x.device)
    p, r = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    y = x.clone()
    y[..., p], y[..., r] = x[..., p] * c - x[..., r] * s, x[..., p] * s + x[..., r] * c
    return y


def draw(B, Hq, Hkv, n, D, seed, norm=True, layout="token"):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    if layout == "token":            # views of a projection's output
        qkv = rn(B, n, Hq + 2 * Hkv, D).to(torch.bfloat16)
        q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    else:                            # head by head, rows with a gap
        q, k = (rn(B, H, n, D + 8).to(torch.bfloat16)[..., :D] for H in (Hq, Hkv))
    w = [1 + 0.2 * rn(D) for _ in range(2)] if norm else [None, None]
    return q, k, w[0], w[1], rn


def reference(x, w, pos, freq, rope):
    y = x.double()
    if w is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + rope.eps) * w.double()
    return turned(y, pos, freq, rope.interleaved, rope.rotary, rope.amplitude or 1.0)


def pair_size(y):
    return y.abs().amax(-1, keepdim=True)


def check(got, ref):
    assert (got.double() - ref).abs().sub(2.0 ** -8 * ref.abs() + 2.0 ** -17 * pair_size(ref)).max() <= 0


CASES = [  # D, Hq, Hkv, B, n, rotary, interleaved, norm, layout
    (128, 8, 2, 1, 1, 128, False, True, "token"), (128, 32, 8, 2, 7, 128, True, True, "token"), (64, 12, 12, 3, 65, 32, False, True, "head"),
    (64, 4, 4, 1, 130, 64, True, False, "token"), (256, 16, 8, 1, 33, 64, False, True, "token"), (256, 4, 2, 2, 100, 256, True, True, "head"),
    (128, 4, 1, 1, 600, 0, False, True, "token"), (128, 4, 2, 2, 40, 0, True, False, "head"), (128, 6, 3, 1, 50, 20, False, True, "token"),
    (64, 3, 1, 2, 19, 2, False, True, "head"), (256, 2, 1, 1, 21, 250, False, True, "token"), (128, 5, 5, 1, 31, 70, True, True, "token"),
    (256, 2, 2, 1, 9, 6, False, False, "token"), (128, 1, 1, 1, 5000, 128, False, True, "head"), (64, 2, 1, 300, 1, 64, False, True, "token"),
    (128, 40, 1, 1, 2500, 96, False, True, "token"),
    # one round of whole tiles and a few behind it, two, five
    (64, 12, 12, 3, 1021, 32, True, True, "token"), (256, 16, 8, 1, 2600, 256, False, True, "head"), (64, 12, 4, 8, 1301, 64, False, True, "token"),
]


@pytest.mark.parametrize("D,Hq,Hkv,B,n,rotary,interleaved,norm,layout", CASES)
def test_forward(D, Hq, Hkv, B, n, rotary, interleaved, norm, layout):
    q, k, wq, wk, rn = draw(B, Hq, Hkv, n, D, D + n, norm, layout)
    rope = fb.make_rope(rotary, interleaved, amplitude=1.25, eps=1e-5)
    freq = fb.focus_rope_frequencies(rotary)[0]
    pos = torch.randint(0, 1 << 20, (B, n), device="cuda", dtype=torch.int32)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16, batch=B)
    for p in (pos, None):
        qo, ko = (torch.full(x.shape, float("nan"), dtype=torch.bfloat16, device="cuda") for x in (q, k))
        fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, p, qo, ko)
        at = p if p is not None else torch.arange(n, device="cuda").expand(B, n)
        check(qo, reference(q, wq, at, freq, rope))
        check(ko, reference(k, wk, at, freq, rope))
    # in place
    q2, k2 = q.clone(), k.clone()
    fb.focus_qk_norm_rope(shape, rope, q2, k2, wq, wk, freq, None, q2, k2)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


def backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk, dq=None, dk=None):
    dq, dk = (torch.full(x.shape, float("nan"), dtype=torch.bfloat16, device="cuda") if d is None else d for x, d in ((q, dq), (k, dk)))
    dwq, dwk = (None if w is None else torch.full_like(w, float("nan")) for w in (wq, wk))
    ws = torch.full((fb.focus_qk_norm_rope_bwd_workspace_bytes(shape),), 0xff, dtype=torch.uint8, device="cuda")
    fb.focus_qk_norm_rope_bwd(shape, rope, q, k, wq, wk, freq, pos, gq, gk, dq, dk, dwq, dwk, ws)
    return dq, dk, dwq, dwk


@pytest.mark.parametrize("D,Hq,Hkv,B,n,rotary,interleaved,norm,layout", CASES)
def test_backward(D, Hq, Hkv, B, n, rotary, interleaved, norm, layout):
    q, k, wq, wk, rn = draw(B, Hq, Hkv, n, D, D + n, norm, layout)
    rope = fb.make_rope(rotary, interleaved, amplitude=0.75, eps=1e-5)
    freq = fb.focus_rope_frequencies(rotary)[0]
    pos = torch.randint(-1000, 1 << 20, (B, n), device="cuda", dtype=torch.int32)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16, batch=B)
    gq, gk = (rn(B, H, n, D).to(torch.bfloat16) for H in (Hq, Hkv))
    dq, dk, dwq, dwk = backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk)
    for x, w, g, dx, dw, H in ((q, wq, gq, dq, dwq, Hq), (k, wk, gk, dk, dwk, Hkv)):
        # the formula, and autograd of the forward definition in 64 bits
        leaf = x.double().requires_grad_()
        wl = None if w is None else w.double().requires_grad_()
        y = reference(leaf, wl, pos, freq, rope)
        grads = torch.autograd.grad(y, [leaf] + ([wl] if wl is not None else []), g.double())
        back = turned(g.double(), pos, freq, interleaved, rotary, 0.75, -1.0)
        if w is None:
            check(dx, back)
        else:
            r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + rope.eps)
            u, xhat = back * w.double(), x.double() * r
            ref = r * (u - xhat * (u * xhat).mean(-1, keepdim=True))
            assert (ref - grads[0]).abs().max() < 1e-10
            size = r * (pair_size(u) + pair_size(xhat) * (u * xhat).abs().mean(-1, keepdim=True))
            assert (dx.double() - ref).abs().sub(2.0 ** -8 * ref.abs() + 2.0 ** -17 * size).max() <= 0
            mag = (pair_size(back) * xhat.abs()).sum((0, 1, 2))
            assert (dw.double() - grads[1]).abs().sub(mag * (2.0 ** -24 * (B * H * n / 8 + 96) + 2.0 ** -18)).max() <= 0
    # the same bits again, and in place of the gradients
    again = backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk)
    inplace = backward(shape, rope, q, k, wq, wk, freq, pos, gq2 := gq.clone(), gk2 := gk.clone(), gq2, gk2)
    for a, b, c in zip((dq, dk, dwq, dwk), again, inplace):
        assert a is None or (torch.equal(a, b) and torch.equal(a, c))


def test_gradients_against_differences():
    """the derivative of sum(g . y) along random directions, by central differences of the forward formula"""
    B, Hq, Hkv, n, D = 1, 4, 2, 9, 64
    q, k, wq, wk, rn = draw(B, Hq, Hkv, n, D, 5)
    rope, freq = fb.make_rope(32, True, eps=1e-3), fb.focus_rope_frequencies(32)[0]
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)[None]
    gq, gk = (rn(B, H, n, D).to(torch.bfloat16) for H in (Hq, Hkv))
    dq, dk, dwq, dwk = backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        f = lambda a, b: (g.double() * reference(a, b, pos, freq, rope)).sum()
        e, v, u = 1e-5, rn(*x.shape).double(), rn(D).double()
        along = (f(x.double() + e * v, w) - f(x.double() - e * v, w)) / (2 * e)
        assert abs(along - (dx.double() * v).sum()) <= 2.0 ** -8 * (dx.double() * v).abs().sum()
        along = (f(x.double(), w.double() + e * u) - f(x.double(), w.double() - e * u)) / (2 * e)
        assert abs(along - (dw.double() * u).sum()) <= 2.0 ** -16 * (dw.double() * u).abs().sum() + 1e-6


def test_rows_of_zeros_large_numbers_and_far_positions():
    n, D = 64, 128
    q, k, wq, wk, rn = draw(1, 2, 1, n, D, 3)
    q, k = q.contiguous(), k.contiguous()
    q[0, 0, 5] = 0
    q[0, 1, 7] *= 1e15
    k[0, 0, 9] *= 1e-15
    rope, freq = fb.make_rope(D), fb.focus_rope_frequencies(D, 500000.0)[0]
    pos = torch.full((1, n), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    pos[0, ::2] = -2 ** 31
    shape = fb.make_shape(2, 1, n, D, 4, 2, 16)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, pos, qo, ko)
    assert qo[0, 0, 5].abs().max() == 0
    check(qo, reference(q, wq, pos, freq, rope))
    check(ko, reference(k, wk, pos, freq, rope))


def test_one_of_the_weights_alone():
    q, k, wq, wk, rn = draw(1, 4, 2, 33, 64, 8)
    rope, freq = fb.make_rope(64), fb.focus_rope_frequencies(64)[0]
    shape = fb.make_shape(4, 2, 33, 64, 4, 2, 16)
    pos = torch.arange(33, device="cuda", dtype=torch.int32)[None]
    gq, gk = (rn(*x.shape).to(torch.bfloat16) for x in (q, k))
    both = backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk)
    only_q = backward(shape, rope, q, k, wq, None, freq, pos, gq, gk)
    only_k = backward(shape, rope, q, k, None, wk, freq, pos, gq, gk)
    assert torch.equal(both[0], only_q[0]) and torch.equal(both[2], only_q[2]) and only_q[3] is None
    assert torch.equal(both[1], only_k[1]) and torch.equal(both[3], only_k[3])
    check(only_q[1], turned(gk.double(), pos, freq, False, 64, 1.0, -1.0))


def test_replay_and_another_stream():
    B, Hq, Hkv, n, D = 2, 8, 2, 100, 128
    q, k, wq, wk, rn = draw(B, Hq, Hkv, n, D, 4)
    rope, freq = fb.make_rope(D), fb.focus_rope_frequencies(D)[0]
    pos = torch.randint(0, 5000, (B, n), device="cuda", dtype=torch.int32)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16, batch=B)
    gq, gk = (rn(*x.shape).to(torch.bfloat16) for x in (q, k))
    outs = [torch.empty(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, k, q, k)] + [torch.empty(D, device="cuda") for _ in range(2)]
    ws = torch.empty(fb.focus_qk_norm_rope_bwd_workspace_bytes(shape), dtype=torch.uint8, device="cuda")

    def call(stream=None):
        fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, pos, outs[0], outs[1], stream)
        fb.focus_qk_norm_rope_bwd(shape, rope, q, k, wq, wk, freq, pos, gq, gk, *outs[2:], ws, stream)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    pos.add_(17)
    gq.neg_()
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in outs]
    for x in outs:
        x.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, outs))


def test_a_large_call():
    """more tiles than the grid, offsets past 2^31 bytes"""
    B, Hq, Hkv, n, D = 1, 32, 8, 140001, 128
    g = torch.Generator(device="cuda"); g.manual_seed(1)
    qkv = torch.randn((B, n, Hq + 2 * Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16)
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    wq, wk = (1 + 0.2 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    rope, freq = fb.make_rope(D), fb.focus_rope_frequencies(D)[0]
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16)
    qo, ko = torch.empty((B, Hq, n, D), dtype=torch.bfloat16, device="cuda"), torch.empty((B, Hkv, n, D), dtype=torch.bfloat16, device="cuda")
    fb.focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, None, qo, ko)
    for rows in (slice(0, 70), slice(70000, 70100), slice(n - 100, n)):
        at = torch.arange(n, device="cuda")[rows][None]
        check(qo[:, :, rows], reference(q[:, :, rows], wq, at, freq, rope))
        check(ko[:, :, rows], reference(k[:, :, rows], wk, at, freq, rope))
    # the derivative: whole rows again, weights by the sum over all of them
    dq, dk, dwq, dwk = backward(shape, rope, q, k, wq, wk, freq, None, qo, ko)
    ref = torch.zeros(D, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(ref)
    for h in range(Hkv):
        x = k[:, h:h + 1].double()
        xhat = x / torch.sqrt(x.square().mean(-1, keepdim=True) + rope.eps)
        back = turned(ko[:, h:h + 1].double(), torch.arange(n, device="cuda")[None], freq, False, D, 1.0, -1.0)
        ref += (back * xhat).sum((0, 1, 2))
        mag += (pair_size(back) * xhat.abs()).sum((0, 1, 2))
    assert (dwk.double() - ref).abs().sub(mag * (2.0 ** -24 * (Hkv * n / 8 / 592 + 200) + 2.0 ** -18)).max() <= 0
    assert dq.isfinite().all() and dk.isfinite().all()
