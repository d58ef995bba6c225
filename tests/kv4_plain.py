"""The 4-bit cache and the attention over it in plain torch, 64 bits: written from the definitions in include/focus.h, by distance to the
numbers that a code and a scale can be."""
import math

import torch

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
SCALES = torch.tensor([e / 512 if e < 8 else (8 + e % 8) * 2.0 ** (e // 8 - 10) for e in range(127)], dtype=torch.float64)


def nearest(y, values):
    """index of the nearest of the ascending `values`, of two equally near ones the even index; beyond the last the last"""
    i = torch.searchsorted(values, y.contiguous()).clamp(1, len(values) - 1)
    lo, hi = y - values[i - 1], values[i] - y
    return torch.where((hi < lo) | ((hi == lo) & (i % 2 == 0)), i, i - 1)


def quantise(x, scale):
    """codes int64 [..., D] and scale codes [..., D / 16] of a CPU tensor x"""
    y = x.double().unflatten(-1, (-1, 16)) / scale
    s = nearest(y.abs().amax(-1) / 6, SCALES) if not x.isnan().any() else None
    v = SCALES[s][..., None]
    a = torch.where(v > 0, y.abs() / torch.where(v > 0, v, torch.ones_like(v)), torch.zeros_like(y))
    c = nearest(a, GRID)
    return (c + 8 * ((y < 0) & (v > 0))).flatten(-2), s


def values(codes, scales, scale):
    v = GRID[codes % 8] * torch.where(codes >= 8, -1.0, 1.0).double()
    return (v.unflatten(-1, (-1, 16)) * (SCALES[scales] * scale)[..., None]).flatten(-2)


def rounded(x, scale):
    """what x stands for in 4 bits"""
    return values(*quantise(x.cpu(), scale), scale)


def attend(q, k, v, keep, scale=None, cap=0.0):
    """q [G, D], k, v [len, D], keep [G, len] -> o [G, D], lse [G], sum p |v|, largest sum |q k| * scale of an attended key"""
    scale = scale or 1 / math.sqrt(q.shape[-1])
    s = q.double() @ k.double().T * scale
    size = q.double().abs() @ k.double().abs().T * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    s = s.masked_fill(~keep, -math.inf)
    p = torch.softmax(s, -1)
    return p @ v.double(), torch.logsumexp(s, -1), p @ v.double().abs(), size.masked_fill(~keep, 0).amax(-1)


def tolerances(o, pv, size, lse, count):
    """What o (bf16) and lse (fp32) may be off by.  A score is an fp32 sum of exact products: at most 16 steps of 16 products, each step
    off by 2^-23 of the sum of magnitudes, and a handful of roundings on the way to the exponential: 2^-18 of that sum, plus 2^-21 of the
    exponent for the fp32 exponentials.  Probabilities are rounded to 11 bits (2^-11), below 2^-24 of the largest to multiples of 2^-35 of it;
    their fp32 sums are off by count / 128 steps a lane (2^-24 each) and a few joins; O is rounded to bf16 (2^-8)."""
    ds = 2.0 ** -18 * (size + 4)
    sums = 2.0 ** -24 * (count / 64 + 64)
    tol_o = 2.0 ** -8 * o.abs() + (2.0 ** -11 + 2 * ds + sums)[..., None] * pv + count * 2.0 ** -35 * 8
    return tol_o, ds + sums + 2.0 ** -22 * lse.abs()
