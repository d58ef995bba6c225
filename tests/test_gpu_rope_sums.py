"""The weight gradients of norm and rotation as sums in which every row counts once.

Exact ones: x is +1 or -1, so that the mean of squares is 1 and (without eps) its root is 1; the frequencies are 0, so that every pair is turned by nothing; the
gradients are odd whole numbers up to 15.  Then a row's term is an odd whole number, all sums stay below 2^24 and are exact in fp32 in any order, and
a pass left out, or one made twice, changes the sums.

Random ones: a term is off by 2^-18 of its size (an angle to 2^-21, the root to 2^-19, a dozen products).  A sum's chain: the passes of a
CTA, the rows of threads (32 at D = 128, 64 at 64, 16 at 256), the CTAs eight at a time from 32 rows of threads (296 / 256 rounds of 8), five
exchanges: `chain` additions of 2^-24 of the sum of magnitudes each."""
import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from tests.test_gpu_rope import backward, turned

pytestmark = pytest.mark.gpu

EXACT = [  # D, Hq, Hkv, B, n: how tiles of tokens, in rounds of one per CTA, come out
    (128, 8, 2, 1, 1), (64, 12, 12, 3, 5), (128, 8, 8, 1, 149), (64, 12, 12, 8, 68), (256, 16, 8, 1, 150),         # a tile per CTA, one pass
    (128, 8, 8, 2, 777), (256, 4, 2, 1, 1301), (256, 64, 1, 1, 333),                                               # fewer tiles than CTAs, several passes
    (64, 12, 12, 3, 1021), (64, 12, 4, 8, 1301), (128, 32, 8, 1, 2501), (256, 16, 8, 1, 2600), (128, 40, 1, 1, 2500),      # a few rounds and tiles behind them
    (128, 32, 8, 1, 8192), (64, 12, 12, 4, 4100), (256, 8, 8, 2, 5003), (128, 2, 1, 1, 30011), (64, 1, 1, 700, 3),         # four and more, and tiles behind them
    (128, 8, 8, 1, 148 * 16), (64, 4, 4, 1, 148 * 64), (128, 16, 16, 4, 1184)]                                     # rounds that come out even


def whole(g, *shape):
    return (2 * torch.randint(-8, 8, shape, generator=g, device="cuda") + 1).to(torch.bfloat16)


@pytest.mark.parametrize("interleaved,rotary", [(False, 1.0), (True, 1.0), (False, 0.0), (False, -1)])
@pytest.mark.parametrize("D,Hq,Hkv,B,n", EXACT)
def test_every_row_counts_once(D, Hq, Hkv, B, n, interleaved, rotary):
    rotary = 6 if rotary < 0 else int(rotary * D)                          # (6: halves that are no whole 16 bytes)
    g = torch.Generator(device="cuda"); g.manual_seed(D + n)
    sign = lambda H: (2 * torch.randint(0, 2, (B, n, H, D), generator=g, device="cuda") - 1).to(torch.bfloat16).transpose(1, 2)
    q, k = sign(Hq), sign(Hkv)
    gq, gk = whole(g, B, Hq, n, D), whole(g, B, Hkv, n, D)
    w = torch.ones(D, device="cuda")
    rope = fb.make_rope(rotary, interleaved, eps=0.0)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 0, batch=B)
    freq = torch.zeros(rotary // 2, dtype=torch.float64, device="cuda")
    dq, dk, dwq, dwk = backward(shape, rope, q, k, w, w, freq, None, gq, gk)
    for x, gx, dw, dx in ((q, gq, dwq, dq), (k, gk, dwk, dk)):
        assert B * x.shape[1] * n * 15 < 1 << 24
        assert torch.equal(dw.double(), (x.double() * gx.double()).sum((0, 1, 2)))
        # and its vector: x (x g - mean(x g)), whole numbers and a mean of 1 / D steps, rounded once
        xg = (x.double() * gx.double())
        ref = x.double() * (xg - xg.mean(-1, keepdim=True))
        assert (dx.double() - ref).abs().sub(2.0 ** -8 * ref.abs() + 2.0 ** -19).max() <= 0


CHAIN = [(64, 12, 12, 3, 1021, 32, True), (64, 12, 4, 8, 1301, 64, False), (256, 16, 8, 1, 2600, 256, False), (128, 32, 8, 1, 8192, 128, False),
         (128, 8, 8, 2, 777, 128, True), (128, 2, 1, 1, 30011, 64, False), (128, 6, 3, 1, 5000, 20, False)]


@pytest.mark.parametrize("D,Hq,Hkv,B,n,rotary,interleaved", CHAIN)
def test_sums_by_the_chain_that_makes_them(D, Hq, Hkv, B, n, rotary, interleaved):
    g = torch.Generator(device="cuda"); g.manual_seed(D + n)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    q, k, gq, gk = (rn(B, H, n, D).to(torch.bfloat16) for H in (Hq, Hkv, Hq, Hkv))
    wq, wk = (1 + 0.2 * rn(D) for _ in range(2))
    rope = fb.make_rope(rotary, interleaved, amplitude=0.75, eps=1e-5)
    freq = fb.focus_rope_frequencies(rotary)[0]
    pos = torch.randint(-1000, 1 << 20, (B, n), generator=g, device="cuda", dtype=torch.int32)
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 16, batch=B)
    _, _, dwq, dwk = backward(shape, rope, q, k, wq, wk, freq, pos, gq, gk)
    odd = not interleaved and rotary % 16 != 0
    for x, gx, dw, H in ((q, gq, dwq, Hq), (k, gk, dwk, Hkv)):
        back = turned(gx.double(), pos, freq, interleaved, rotary, 0.75, -1.0)
        xhat = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + rope.eps)
        # a term's size: an angle's error moves a number by that of its partner (16 bits of both are in the row's pair)
        p = torch.arange(D, device="cuda")
        half = rotary // 2
        partner = torch.where(p >= rotary, p, (p ^ 1) if interleaved else (p + half) % max(rotary, 1))
        size = ((back.abs() + back.abs()[..., partner]) * xhat.abs()).sum((0, 1, 2))
        # CTAs of a side: its share of 296 (592 for the odd halves) by heads
        ctas = (592 if odd else 296) * H // (Hq + Hkv)
        rows = 8 if odd else 256 * 16 // D                                 # rows of a pass: of one token, or of 2, 4, ... 16
        if odd:
            terms = -(-B * n // (8 * ctas)) * H                            # of a lane
        else:                                                              # the tokens of a tile are chosen by about this sum; a CTA has a tile more or less
            terms = 8 + min(-(-B * -(-n // T) * -(-H // (rows // T)) // ctas) + -(-B * -(-n // T) // ctas) for T in (1, 2, 4, 8, 16) if T == 1 or T * H <= 8 * rows)
        chain = terms + rows + 8 * -(-592 // 256) + 5
        assert (dw.double() - (back * xhat).sum((0, 1, 2))).abs().sub(size * (2.0 ** -24 * chain + 2.0 ** -18)).max() <= 0
