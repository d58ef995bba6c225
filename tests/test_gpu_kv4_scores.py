"""The 4-bit decode step at the ends of the range of scores, against 64 bits.

Keys and queries are such that a score's sum is exact: the query has two numbers that are not 0, the key's are codes.  What is left of the
way to O: the scores' factor (three fp32 roundings, 2^-22 of an exponent's difference from the largest, which is below 2^9 where the
probability is not 0: 2^-12 of it, of one sign for all keys), the exponential (2^-21), fp16 probabilities (2^-11; at 2^-24 of the largest and
below multiples of 2^-35), fp32 sums (2^-17 in all), O rounded to bf16 (2^-8)."""
import math

import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from tests.test_gpu_kv4 import compare, decode, filled, gen, pool, status, stored, table_of

pytestmark = pytest.mark.gpu


def two_numbers(D, steps, big, small, scale, attended, cap=0.0, seed=1):
    """One head, keys (3, steps[j] / 2, 0, ...) and a query (big, small, 0, ...): scores 3 big + steps[j] / 2 small.  The newest key, which is always
    attended, lies far below.  (o, lse, o in 64 bits, the sum of p |v| there, lse in 64 bits)"""
    n = len(steps) + 1
    g = gen(seed)
    shape = fb.make_shape(1, 1, n, D, 4, 1, 0, scale, cap)
    table, num = table_of([n], 64)
    cache = pool(shape, 64, table, num, [n])
    k = torch.zeros((1, 1, n, D), device="cuda")
    k[..., 0] = 3.0
    k[0, 0, :-1, 1] = steps / 2
    k[0, 0, -1, 0] = -3.0
    v = torch.randn((1, 1, n, D), generator=g, device="cuda").to(torch.bfloat16)
    mk = torch.zeros((1, n), dtype=torch.int32, device="cuda")
    mk[0, :-1] = attended.int()
    st = status()
    fb.focus_kv4_append(shape, cache, k.to(torch.bfloat16), v, mk, None, st)
    ks, vs = stored(cache, 1, D, n)
    assert torch.equal(ks.float(), k) and st[0].item() == 0
    q = torch.zeros((1, 1, D), device="cuda")
    q[..., 0], q[..., 1] = big, small
    q = q.to(torch.bfloat16)
    assert q[0, 0, 0].item() == big and q[0, 0, 1].item() == small
    o, lse = decode(cache, shape, q, torch.ones(1, dtype=torch.int32, device="cuda"))
    s = (ks[0, 0].double() @ q[0, 0].double()) * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    keep = torch.cat([attended, torch.ones(1, dtype=torch.bool, device="cuda")])
    s = s.masked_fill(~keep, -math.inf)
    p = torch.softmax(s, -1)
    return o[0, 0].double(), lse[0, 0].double(), p @ vs[0, 0].double(), p @ vs[0, 0].double().abs(), torch.logsumexp(s, -1)


# (the scale that is asked for is rounded to fp32 on its way: powers of two)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lg", [-10, 0, 4, 8, 10, 12, 20, 40, 60, 80])
def test_large_scores_a_few_units_apart(D, lg):
    """Scores of 3 * 2^13 * 2^lg and of up to twelve fp32 units more: at 2^24 and beyond a unit is several powers of e.  All attended keys are one warp's, so
    that the reference that probabilities are taken to is set by the first tile and outrun, by less than its headroom or by more, by the next."""
    tile = 16 if D == 256 else 32
    far = 4 * tile                                     # (a warp has a quarter of the keys, in whole tiles)
    n = 4 * far
    for order in (1, -1):
        steps = torch.zeros(n - 1, device="cuda")
        steps[:far] = torch.arange(far, device="cuda") // tile * (2.0 * order) + (4.0 if order < 0 else 0.0)      # key numbers 0 to 3
        steps = (steps - steps.min()).clamp(0, 12)
        # numbers that a block of scale 1 / 2 can hold beside 3: 0, 1, 2, 3
        attended = torch.arange(n - 1, device="cuda") < far
        o, lse, ro, pv, rl = two_numbers(D, steps, 2.0 ** 13, 2.0 ** -9, 2.0 ** lg, attended)
        assert o.isfinite().all() and lse.isfinite()
        tol = 2.0 ** -8 * ro.abs() + (2.0 ** -11 + 2 * (2.0 ** -12 + 2.0 ** -21) + 2.0 ** -17) * pv + n * 2.0 ** -35 * 8
        assert (o - ro).abs().sub(tol).max() <= 0, (o - ro).abs().max()
        assert (lse - rl).abs() <= 2.0 ** -21 * rl.abs() + 2.0 ** -11


@pytest.mark.parametrize("cap", [2.0 ** 20, 2.0 ** 30])
def test_large_cap(cap):
    """a cap far beyond the scores is none: tanh of a small number, times the cap, is off by a few fp32 units"""
    D, n = 128, 4 * 128
    steps = (torch.arange(n - 1, device="cuda") // 32 * 2.0).clamp(max=6)
    o, lse, ro, pv, rl = two_numbers(D, steps, 2.0 ** -4, 2.0 ** -6, 1.0, torch.ones(n - 1, dtype=torch.bool, device="cuda"), cap)
    tol = 2.0 ** -8 * ro.abs() + (2.0 ** -11 + 2.0 ** -18) * pv + n * 2.0 ** -35 * 8
    assert (o - ro).abs().sub(tol).max() <= 0 and (lse - rl).abs() <= 2.0 ** -17


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 1.0, 2.0 ** -140])
@pytest.mark.parametrize("lg", [-120, -60, -24, 0])
def test_queries_of_zeros_and_scales_near_nothing(D, cap, lg):
    """All scores are 0 (or too small to tell from it): o is the mean of the attended values, and the others have no weight."""
    lens, Hq, Hkv = [700, 33, 1], 4, 2
    cache, q, mq, mk, k, v = filled(lens, 32, Hq, Hkv, D, 8, 1, D)
    pages, table, dl = cache.tensors
    cache = fb.make_kv4(pages, 32, table, dl, 2.0 ** -16, 2.0)       # (the codes as they are, for keys 2^15 times smaller)
    q[:, ::2] = 0
    q *= 2.0 ** -40
    shape = fb.make_shape(Hq, Hkv, 700, D, 8, 1, 5, 2.0 ** lg, cap, batch=3)
    o, lse = decode(cache, shape, q, mq)
    ks, vs = stored(cache, Hkv, D, 700)
    compare(o, lse, lens, q, mq, mk, ks, vs, 5, cap, 2.0 ** lg)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_the_largest_queries_and_scales_over_keys_of_zeros(D, cap):
    """scores are 0 however large what they are multiplied by: the factor stays a number"""
    lens, Hq, Hkv, n = [300], 4, 2, 300
    cache, q, mq, mk, k, v = filled(lens, 32, Hq, Hkv, D, 4, 1, D)
    pages, table, dl = cache.tensors
    cache = fb.make_kv4(pages, 32, table, dl, 2.0 ** 16, 1.0)
    fb.focus_kv4_append(fb.make_shape(Hq, Hkv, n, D, 4, 1, 0), cache, torch.zeros_like(k), v, mk)
    q.fill_(torch.finfo(torch.bfloat16).max)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 1, 3, 2.0 ** 20, cap)
    o, lse = decode(cache, shape, q, mq)
    ks, vs = stored(cache, Hkv, D, n)
    assert (ks == 0).all()
    compare(o, lse, lens, torch.zeros_like(q), mq, mk, ks, vs, 3)
