"""focus_router_scores_bwd with many groups and long centroids (the folded projection by a launch of its own), and with what is not finite."""
import math

import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from test_gpu_router_bwd import bounds, call, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,n,d,dg,K", [(1, 300, 1024, 128, 32), (1, 65, 40, 33, 17), (2, 200, 264, 64, 24), (1, 1, 64, 513, 31), (1, 500, 2056, 65, 16), (1, 900, 4096, 200, 32)])
def test_many_groups(B, n, d, dg, K):
    h, Wg, C, ds = inputs(B, n, d, dg, K, n + d + K)
    shape = fb.make_shape(1, 1, n, 64, K, 1, 0, batch=B)
    for got, (want, bound) in zip(call(shape, h, Wg, C, ds), bounds(h, Wg, C, ds, K)):
        assert ((got.double() - want).abs() <= bound + 1e-30).all(), ((got.double() - want).abs() / bound).max().item()


@pytest.mark.parametrize("K,dg", [(4, 16), (8, 16), (16, 8), (32, 128)])
def test_where_groups_cancel(K, dg):
    """centroids that differ little and gradients that sum to nearly nothing: dh is right to 2^-14 of the magnitudes, as ever, and no better: dscores and the
    folded projection have 16 bits each in it"""
    n, d = 300, 256
    h, Wg, C, ds = inputs(1, n, d, dg, K, K)
    C = C[:1] + 1e-3 * C
    ds[..., :K] -= ds[..., :K].mean(-1, keepdim=True)
    for got, (want, bound) in zip(call(fb.make_shape(1, 1, n, 64, K, 1, 0), h, Wg, C, ds), bounds(h, Wg, C, ds, K)):
        assert ((got.double() - want).abs() <= bound + 1e-30).all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("K", [3, 8, 20])
def test_what_is_not_finite_stays_where_it_belongs(bad, K):
    n, d, dg, token, col, group = 200, 128, 16, 77, 41, 1
    h, Wg, C, ds = inputs(1, n, d, dg, K, 5)
    shape = fb.make_shape(1, 1, n, 64, K, 1, 0)
    dh, dWg, dC = call(shape, h, Wg, C, ds)
    # in h: that column of dW_g, and dC, which sums over all columns
    h[0, token, col] = bad
    a, b, c = call(shape, h, Wg, C, ds)
    keep = torch.arange(d, device="cuda") != col
    assert torch.equal(a, dh) and torch.equal(b[keep], dWg[keep]) and not b[col].isfinite().any() and not c[:K].isfinite().any()
    # in the scores' gradient: that token's dh, that group's dC, and dW_g, which sums over all groups
    h, Wg, C, ds = inputs(1, n, d, dg, K, 5)
    ds[0, token, group] = bad
    a, b, c = call(shape, h, Wg, C, ds)
    keep, rows = torch.arange(K, device="cuda") != group, torch.arange(n, device="cuda") != token
    assert torch.equal(a[0, rows], dh[0, rows]) and not a[0, token].isfinite().any() and torch.equal(c[keep], dC[keep]) and not c[group].isfinite().any()
    assert not b.isfinite().any()
