"""focus_router_scores_bwd against the formula in 64 bits (the chain from a loss to the router's weights: test_gpu_gate_layer.py)."""
import math

import pytest
import torch

import bwd_plain as plain
from paper_2604_03260_b200 import binding as fb

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
# sums over N tokens in fp32, 2^-24 of the absolute terms for each of some hundred steps in a row at most (pieces of 32 tokens, runs, blocks of runs),
# twice over for the two products, and the lost ends of bf16 terms
E = 2.0 ** -14


def inputs(B, n, d, dg, K, seed, pad=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    h = torch.randn((B, n, d + pad), generator=gen, device="cuda").to(torch.bfloat16)[..., :d]
    Wg, C = torch.randn((d, dg), generator=gen, device="cuda") / math.sqrt(d), torch.randn((K, dg), generator=gen, device="cuda")
    ds = torch.randn((B, n, fb.focus_soft_ld(K)), generator=gen, device="cuda")
    return h, Wg, C, ds


def call(shape, h, Wg, C, ds, dh="new", stream=None):
    dh = torch.full_like(h, math.nan) if isinstance(dh, str) else dh
    dWg, dC = torch.full_like(Wg, math.nan), torch.full_like(C, math.nan)
    ws = torch.empty(fb.focus_router_scores_bwd_workspace_bytes(shape, h.shape[-1], Wg.shape[1]), dtype=torch.uint8, device="cuda").fill_(0xff)
    fb.focus_router_scores_bwd(shape, h, Wg, C, ds, dh, dWg, dC, ws, stream)
    torch.cuda.synchronize()
    return dh, dWg, dC


def bounds(h, Wg, C, ds, K):
    """(value, bound) of dh, dWg, dC"""
    s, x, W, c = ds[..., :K].double().flatten(0, 1), h.double().flatten(0, 1), Wg.double(), C.double()
    dh = (s @ (c @ W.T)).view(h.shape)
    eh = U * dh.abs() + E * (s.abs() @ (c.abs() @ W.abs().T)).view(h.shape)
    T, aT = s.T @ x, s.abs().T @ x.abs()
    return (dh, eh), (T.T @ c, E * (aT.T @ c.abs())), (T @ W, E * (aT @ W.abs()))


@pytest.mark.parametrize("B,n,d,dg,K", [(1, 1, 8, 1, 1), (1, 3, 64, 16, 4), (2, 127, 72, 5, 3), (1, 128, 512, 16, 4), (3, 129, 768, 16, 8), (1, 1000, 520, 16, 7), (2, 700, 1024, 33, 16),
                                        (1, 5000, 136, 16, 32), (1, 300, 4096, 128, 8), (1, 257, 2056, 16, 20), (4, 33, 256, 300, 5), (1, 20000, 256, 16, 8)])
def test_against_the_formula(B, n, d, dg, K):
    h, Wg, C, ds = inputs(B, n, d, dg, K, n + d)
    shape = fb.make_shape(1, 1, n, 64, K, 1, 0, batch=B)
    for got, (want, bound) in zip(call(shape, h, Wg, C, ds), bounds(h, Wg, C, ds, K)):
        assert ((got.double() - want).abs() <= bound + 1e-30).all(), ((got.double() - want).abs() / bound).max().item()


def test_padded_rows_in_place_and_without_dh():
    B, n, d, dg, K = 2, 200, 264, 16, 5
    h, Wg, C, ds = inputs(B, n, d, dg, K, 1, pad=24)
    shape = fb.make_shape(1, 1, n, 64, K, 1, 0, batch=B)
    (dh, eh), w, c = bounds(h, Wg, C, ds, K)
    a = call(shape, h.contiguous(), Wg, C, ds)
    b = call(shape, h, Wg, C, ds, None)
    assert b[0] is None and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    whole = torch.full((B, n, d + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    call(shape, h, Wg, C, ds, whole[..., :d])
    assert torch.equal(whole[..., :d], a[0]) and (whole[..., d:] == 3.0).all()
    x = h.contiguous()
    e = call(shape, x, Wg, C, ds, x)
    assert torch.equal(x, a[0]) and torch.equal(e[1], a[1]) and torch.equal(e[2], a[2])


def test_ignored_columns_may_hold_anything():
    h, Wg, C, ds = inputs(1, 150, 128, 8, 3, 2)
    shape = fb.make_shape(1, 1, 150, 64, 3, 1, 0)
    a = call(shape, h, Wg, C, ds)
    ds[..., 3:] = math.nan
    assert all(torch.equal(x, y) for x, y in zip(a, call(shape, h, Wg, C, ds)))


def test_captured_on_a_stream():
    h, Wg, C, ds = inputs(1, 400, 256, 16, 4, 3)
    h2, _, _, ds2 = inputs(1, 400, 256, 16, 4, 4)
    shape = fb.make_shape(1, 1, 400, 64, 4, 1, 0)
    dh, dWg, dC = torch.empty_like(h), torch.empty_like(Wg), torch.empty_like(C)
    ws = torch.empty(fb.focus_router_scores_bwd_workspace_bytes(shape, 256, 16), dtype=torch.uint8, device="cuda")
    fb.focus_router_scores_bwd(shape, h, Wg, C, ds, dh, dWg, dC, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.focus_router_scores_bwd(shape, h, Wg, C, ds, dh, dWg, dC, ws)
    want = call(shape, h2, Wg, C, ds2)
    h.copy_(h2), ds.copy_(ds2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dh, dWg, dC), want))


def test_long_sums_stay_in_32_bits():
    """32768 tokens whose terms all have one sign.  A sum of 32 tokens on the tensor cores is six steps, each cut off by less than 2^-23 of what it has
    by then (a half and the whole of the piece: 4.5 2^-23 at most, taken as six); pieces, parts and columns are added with roundings of half a step,
    2^-24 of the running sum at most and of both signs, some 40 + 4 + 8 of them on average halfway up: below 2^-22 together.  In all below 2^-20."""
    n, d, dg, K = 32768, 4096, 16, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    rnd = lambda *s: 1 + 0.25 * torch.rand(s, generator=gen, device="cuda")
    h, Wg, C, ds = rnd(1, n, d).to(torch.bfloat16), rnd(d, dg), rnd(K, dg), rnd(1, n, K)
    _, dWg, dC = call(fb.make_shape(2, 1, n, 64, K, 1, 0), h, Wg, C, ds, None)
    T = sum(ds[0, i:i + 4096].double().T @ h[0, i:i + 4096].double() for i in range(0, n, 4096))
    for got, want in ((dWg, T.T @ C.double()), (dC, T @ Wg.double())):
        assert (got.double() - want).norm() <= 2.0 ** -20 * want.norm(), ((got.double() - want).norm() / want.norm()).item()
