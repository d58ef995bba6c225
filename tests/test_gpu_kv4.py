"""The 4-bit cache: what goes in comes out as the definition says, bit for bit; the decode step over it against attention in 64 bits on the
numbers that the codes stand for (tolerances derived in kv4_plain.tolerances)."""
import math

import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200.kv4_cache import Kv4Cache
from tests import kv4_plain as kp

pytestmark = pytest.mark.gpu
KS, VS = 0.5, 2.0


def gen(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    return g


def table_of(lens, P, spare=3, seed=0, extra=0):
    """pages in random order: table [B, most], number of pages"""
    most = max(1, max(-(-l // P) for l in lens)) + extra
    need = sum(-(-l // P) for l in lens)
    order = torch.randperm(need + spare, generator=torch.Generator().manual_seed(seed))
    t = torch.full((len(lens), most), -7, dtype=torch.int32)          # entries behind the last page are not read
    at = 0
    for b, l in enumerate(lens):
        m = -(-l // P)
        t[b, :m] = order[at:at + m].to(torch.int32)
        at += m
    return t.cuda(), need + spare


def pool(shape, P, table, num, lens, fill=0xff):
    pages = torch.full((num, fb.focus_kv4_page_bytes(shape, P)), fill, dtype=torch.uint8, device="cuda")
    return fb.make_kv4(pages, P, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), KS, VS)


def status():
    return torch.zeros(4, dtype=torch.int32, device="cuda")


def row_bytes(cache, shape, b, h, pos):
    """codes of key and value, scales, mask of a token, from the raw page"""
    P, D, H = cache.page_tokens, shape.D, shape.Hkv
    pages, table, _ = cache.tensors
    page, at = pages[table[b, pos // P]].cpu(), h * P + pos % P
    c = page[at * D:(at + 1) * D].long()
    c = torch.stack([c % 16, c // 16], -1).flatten()
    s = page[H * P * D + at * (D // 8):][:D // 8].long()
    m = page[H * P * (D + D // 8) + 4 * at:][:4].clone().view(torch.int32).item()
    return c[:D], c[D:], s[:D // 16], s[D // 16:], m


@pytest.mark.parametrize("D,Hkv,P,lens,n,counts", [
    (128, 2, 16, [1], 1, None), (128, 3, 64, [70, 64, 65], 10, None), (64, 4, 32, [33, 200, 7], 7, [0, 7, 3]), (256, 1, 128, [130, 129], 129, [130 - 1, 128]),
    (64, 1, 16, [17], 17, [16]), (256, 5, 256, [300], 300, None), (128, 8, 16, [1000, 5, 16], 5, [5, 5, 0])])
def test_append_and_read(D, Hkv, P, lens, n, counts):
    B, g = len(lens), gen(D + n)
    shape = fb.make_shape(Hkv, Hkv, n, D, 4, 2, 16, batch=B)
    table, num = table_of(lens, P)
    cache = pool(shape, P, table, num, lens)
    pages = cache.tensors[0]
    qkv = (torch.randn((B, n, 3, Hkv, D), generator=g, device="cuda") * torch.exp(torch.randn((B, n, 3, Hkv, 1), generator=g, device="cuda"))).to(torch.bfloat16)
    k, v = qkv[:, :, 1].transpose(1, 2), qkv[:, :, 2].transpose(1, 2)             # token-major views
    mk = torch.randint(-2 ** 31, 2 ** 31 - 1, (B * Hkv, n), generator=g, device="cuda", dtype=torch.int32)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    st = status()
    fb.focus_kv4_append(shape, cache, k, v, mk, cnt, st)
    counts = counts or [n] * B
    assert st.tolist() == [0] * 4
    kr, vr = kp.rounded(k, KS), kp.rounded(v, VS)
    # raw bytes of the first and last tokens, and of all others that nothing changed
    touched = torch.zeros(pages.shape, dtype=torch.bool)
    for b in range(B):
        for t in range(counts[b]):
            pos = lens[b] - counts[b] + t
            p, at = table[b, pos // P].item(), pos % P
            for h in range(Hkv):
                r = h * P + at
                touched[p, r * D:(r + 1) * D] = True
                touched[p, Hkv * P * D + r * (D // 8):][:D // 8] = True
                touched[p, Hkv * P * (D + D // 8) + 4 * r:][:4] = True
            if t in (0, counts[b] - 1):
                for h in range(Hkv):
                    kc, vc, ks, vs, m = row_bytes(cache, shape, b, h, pos)
                    (rk, sk), (rv, sv) = kp.quantise(k[b, h, t].cpu(), KS), kp.quantise(v[b, h, t].cpu(), VS)
                    assert torch.equal(ks, sk) and torch.equal(vs, sv) and m == mk[b * Hkv + h, t].item()
                    # (the sign of a zero is free)
                    assert torch.equal(kc * (kc != 8), rk * (rk != 8)) and torch.equal(vc * (vc != 8), rv * (rv != 8))
    assert (pages.cpu()[~touched] == 0xff).all()
    # back: rows behind the last token stay as they were
    m = n + 3
    big = fb.make_shape(Hkv, Hkv, m, D, 4, 2, 16, batch=B)
    first = torch.tensor([l - c for l, c in zip(lens, counts)], dtype=torch.int32, device="cuda")
    ko, vo = (torch.full((B, m, Hkv, D), 7.0, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
    mo = torch.full((B * Hkv, m), 77, dtype=torch.int32, device="cuda")
    fb.focus_kv4_read(big, cache, first, ko, vo, mo, st)
    assert st.tolist() == [0] * 4
    for b in range(B):
        c = counts[b]
        assert torch.equal(ko[b, :, :c].double().cpu(), kr[b, :, :c]) and torch.equal(vo[b, :, :c].double().cpu(), vr[b, :, :c])
        assert torch.equal(mo.view(B, Hkv, m)[b, :, :c], mk.view(B, Hkv, n)[b, :, :c])
        assert (ko[b, :, c:] == 7).all() and (vo[b, :, c:] == 7).all() and (mo.view(B, Hkv, m)[b, :, c:] == 77).all()


def test_numbers_at_the_edges_of_the_format():
    """ties, zeros, denormal and huge numbers, infinities and NaN"""
    D, H, n, P = 128, 2, 64, 64
    g = gen(1)
    k = (torch.randint(-96, 97, (1, H, n, D), generator=g, device="cuda") / 16).to(torch.bfloat16)          # many ties
    v = torch.randn((1, H, n, D), generator=g, device="cuda").to(torch.bfloat16)
    k[0, 0, 0] = 0
    k[0, 0, 1] *= 1e30
    k[0, 0, 2] *= 1e-30
    k[0, 0, 3] = 2.0 ** -11
    k[0, 0, 4, :16] = torch.finfo(torch.bfloat16).max
    v[0, 1, 5] *= 1e-4
    k[0, 0, 10, 77] = float("nan")
    v[0, 1, 11, 3] = float("-inf")
    v[0, 0, 12, 127] = float("inf")
    shape = fb.make_shape(H, H, n, D, 4, 2, 16)
    table, num = table_of([n], P)
    cache = pool(shape, P, table, num, [n])
    mk = torch.zeros((H, n), dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    fb.focus_kv4_append(shape, cache, k, v, mk)
    fb.focus_kv4_read(shape, cache, None, ko, vo)
    gone = torch.zeros((H, n), dtype=torch.bool)
    for h, t in ((0, 10), (1, 11), (0, 12)):
        gone[h, t] = True
        assert ko[0, h, t].isnan().all() and vo[0, h, t].isnan().all()
    k, v = k.cpu()[0], v.cpu()[0]
    assert torch.equal(ko[0].double().cpu()[~gone], kp.rounded(k[~gone], KS)) and torch.equal(vo[0].double().cpu()[~gone], kp.rounded(v[~gone], VS))


def filled(lens, P, Hq, Hkv, D, K, topk, seed, extra=0, spread=1.0):
    """a cache of random tokens with its keys and values as they stand there, masks, queries"""
    B, g, n = len(lens), gen(seed), max(max(lens), 1)
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, 0, batch=B)
    table, num = table_of(lens, P, seed=seed, extra=extra)
    cache = pool(shape, P, table, num, lens)
    k, v = (torch.randn((B, Hkv, n, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    k *= spread
    masks = lambda *s: ((torch.rand(s + (K,), generator=g, device="cuda").argsort(-1) < topk).int() << torch.arange(K, device="cuda", dtype=torch.int32)).sum(-1).to(torch.int32)
    mk, mq = masks(B * Hkv, n), masks(B * Hq)
    st = status()
    fb.focus_kv4_append(shape, cache, k, v, mk, cache.tensors[2], st)              # (the first lens[b] rows)
    assert st[0].item() == 0
    q = torch.randn((B, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    return cache, q, mq, mk, k, v


def decode(cache, shape, q, mq, ws=None, st=None):
    B, Hq, D = q.shape
    o = torch.full((B, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B * Hq,), float("nan"), device="cuda")
    if ws is None:
        ws = torch.full((fb.focus_kv4_decode_workspace_bytes(shape),), 0xff, dtype=torch.uint8, device="cuda")
    fb.focus_kv4_decode_step(shape, cache, q, mq, o, lse, ws, st)
    return o, lse.view(B, Hq)


def stored(cache, Hkv, D, n):
    """keys and values as they stand in the cache"""
    B = cache.tensors[2].shape[0]
    shape = fb.make_shape(Hkv, Hkv, n, D, 4, 2, 0, batch=B)
    k, v = (torch.zeros((B, Hkv, n, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fb.focus_kv4_read(shape, cache, None, k, v)
    return k, v


def compare(o, lse, lens, q, mq, mk, k, v, window, cap=0.0, scale=0.0, heads=None):
    """k, v as stored, [B, Hkv, n, D]"""
    B, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    mk = mk.view(B, Hkv, -1)
    for b, m in enumerate(lens):
        if m == 0:
            assert (o[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        j = torch.arange(m, device="cuda")
        for h in range(Hkv):
            hs = slice(h * G, (h + 1) * G)
            keep = (m - 1 - j <= window)[None] | ((mk[b, h, None, :m] & mq.view(B, Hq)[b, hs, None]) != 0)
            ro, rl, pv, size = kp.attend(q[b, hs], k[b, h, :m], v[b, h, :m], keep, scale or None, cap)
            tol_o, tol_l = kp.tolerances(ro, pv, size, rl, m)
            assert (o[b, hs].double() - ro).abs().sub(tol_o).max() <= 0, (b, h, (o[b, hs].double() - ro).abs().max())
            assert (lse[b, hs].double() - rl).abs().sub(tol_l).max() <= 0, (b, h, (lse[b, hs].double() - rl).abs().max())


RAGGED = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300, 1000, 0, 513]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,lens,P,K,topk,w", [
    (4, 2, [1], 16, 4, 2, 0), (2, 2, RAGGED, 16, 4, 1, 5), (8, 1, RAGGED, 64, 8, 1, 0), (12, 4, RAGGED, 32, 4, 2, 40), (5, 1, [777], 128, 32, 1, 3),
    (14, 2, [2049, 2048], 256, 4, 2, 3000), (1, 1, [4097], 64, 1, 1, 0), (16, 8, [8200], 64, 8, 2, 100), (2, 2, [9001, 500], 16, 4, 2, 7),
    (3, 3, [5000, 77], 32, 8, 4, 1)])
def test_decode(D, Hq, Hkv, lens, P, K, topk, w):
    cache, q, mq, mk, k, v = filled(lens, P, Hq, Hkv, D, K, topk, D + Hq)
    n = max(lens)
    shape = fb.make_shape(Hq, Hkv, n, D, K, topk, w, batch=len(lens))
    st = status()
    o, lse = decode(cache, shape, q, mq, st=st)
    assert st[0].item() == 0
    ks, vs = stored(cache, Hkv, D, n)
    compare(o, lse, lens, q, mq, mk, ks, vs, w)
    # the same bits again
    o2, lse2 = decode(cache, shape, q, mq)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("D,cap,scale", [(256, 50.0, 0.0), (128, 5.0, 0.25), (64, 0.0, 0.5)])
def test_decode_softcap_and_scale(D, cap, scale):
    lens = [700, 33]
    cache, q, mq, mk, k, v = filled(lens, 32, 8, 4, D, 4, 1, 3)
    shape = fb.make_shape(8, 4, 700, D, 4, 1, 20, scale, cap, batch=2)
    o, lse = decode(cache, shape, q, mq)
    compare(o, lse, lens, q, mq, mk, *stored(cache, 4, D, 700), 20, cap, scale)


@pytest.mark.parametrize("batch,Hq,Hkv,most,D", [(150, 4, 4, 90, 128), (40, 8, 8, 700, 64), (600, 2, 1, 40, 128), (3, 8, 2, 30000, 128), (9, 16, 2, 9000, 256), (1024, 2, 2, 20, 64),
                                                   (32, 4, 2, 257, 128), (33, 4, 2, 256, 64), (128, 8, 8, 300, 128), (129, 2, 2, 500, 256), (500, 1, 1, 255, 128),
                                                   (128, 16, 2, 100, 128), (5, 8, 8, 256, 256), (97, 4, 1, 2000, 64)])
def test_decode_ranges_across_heads(batch, Hq, Hkv, most, D):
    """ranges of the list of units that cover several heads and sequences, end inside one, or are whole ones"""
    g = torch.Generator().manual_seed(batch)
    lens = (torch.rand(batch, generator=g) ** 3 * most).int().tolist()
    lens[0] = most
    cache, q, mq, mk, k, v = filled(lens, 16, Hq, Hkv, D, 4, 1, batch)
    shape = fb.make_shape(Hq, Hkv, most, D, 4, 1, 9, batch=batch)
    o, lse = decode(cache, shape, q, mq)
    ks, vs = stored(cache, Hkv, D, most)
    pick = sorted({0, 1, 2, 7, batch // 2, batch - 1} & set(range(batch)))
    sub = lambda x: x[pick]
    compare(sub(o), sub(lse), [lens[b] for b in pick], sub(q), sub(mq.view(batch, Hq)), sub(mk.view(batch, Hkv, -1)), sub(ks), sub(vs), 9)
    empty = torch.tensor(lens) == 0
    assert (o.cpu()[empty] == 0).all() and (lse.cpu()[empty] == -math.inf).all() and o.isfinite().all()


@pytest.mark.parametrize("bound", [0, 5000])
@pytest.mark.parametrize("D,batch,Hkv,most", [(128, 1, 8, 512), (128, 1, 8, 513), (64, 4, 8, 1024), (64, 4, 8, 1025), (256, 3, 2, 256), (256, 3, 2, 257), (256, 4, 8, 512),
                                              (256, 5, 8, 513), (128, 6, 2, 256), (128, 32, 2, 257), (64, 31, 1, 128), (256, 7, 2, 128), (256, 32, 4, 129), (128, 2, 1, 1)])
def test_decode_heads_of_one_cta(D, batch, Hkv, most, bound):
    """the longest lengths of which a head is left whole, and the first that is not, by the bound of the call or by the lengths"""
    lens = [most if b % 3 == 0 else (37 * b) % (most + 1) for b in range(batch)]
    Hq = 2 * Hkv
    cache, q, mq, mk, k, v = filled(lens, 16, Hq, Hkv, D, 4, 2, most + batch, extra=bound // 16 + 1)
    shape = fb.make_shape(Hq, Hkv, most + bound, D, 4, 2, 9, batch=batch)
    o, lse = decode(cache, shape, q, mq)
    compare(o, lse, lens, q, mq, mk, *stored(cache, Hkv, D, most), 9)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("P,run,hole", [(16, 200, 0.0), (64, 37, 0.2), (128, 700, 0.22), (32, 5, 0.0)])
def test_decode_runs_and_holes(D, P, run, hole):
    """groups in runs of tokens: stretches that no head attends, tiles of 16 or 32 keys that are taken whole although some of their keys are
    not attended (and hold infinities), and single keys between them"""
    lens, Hq, Hkv, K = [20011, 3000], 2, 1, 8
    g = gen(run + D)
    n = max(lens)
    shape = fb.make_shape(Hq, Hkv, n, D, K, 1, 33, batch=2)
    table, num = table_of(lens, P, seed=run)
    cache = pool(shape, P, table, num, lens)
    k, v = (torch.randn((2, Hkv, n, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    group = (torch.arange(n, device="cuda") // run * 5) % K
    mk = (1 << group).to(torch.int32).repeat(2 * Hkv, 1)
    holes = torch.rand(mk.shape, generator=g, device="cuda") < hole
    mk[holes] = 0
    mq = torch.tensor([1, 4, 8, 8], dtype=torch.int32, device="cuda")
    far = torch.stack([torch.arange(n, device="cuda") < m - 1 - 33 for m in lens])
    bad = holes.view(2, Hkv, n) & far[:, None]                      # attended by nobody
    k[bad], v[bad] = float("inf"), float("nan")
    st = status()
    fb.focus_kv4_append(shape, cache, k, v, mk, cache.tensors[2], st)
    q = torch.randn((2, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    o, lse = decode(cache, shape, q, mq, st=st)
    assert st[0].item() == 0
    ks, vs = stored(cache, Hkv, D, n)
    compare(o, lse, lens, q, mq, mk, ks.nan_to_num(), vs.nan_to_num(), 33)


def test_decode_long_cache_and_large_scores():
    lens = [131072]
    cache, q, mq, mk, k, v = filled(lens, 64, 4, 1, 128, 4, 2, 7, spread=6.0)
    shape = fb.make_shape(4, 1, 131072, 128, 4, 2, 100)
    o, lse = decode(cache, shape, q, mq)
    compare(o, lse, lens, q, mq, mk, *stored(cache, 1, 128, 131072), 100)


def test_queries_of_all_magnitudes():
    lens = [200]
    cache, q, mq, mk, k, v = filled(lens, 64, 8, 1, 128, 4, 4, 9)
    for i, f in enumerate((0.0, 1e-38, 1e-20, 1e-6, 1.0, 30.0)):
        q[0, i] *= f
    shape = fb.make_shape(8, 1, 200, 128, 4, 4, 0)
    o, lse = decode(cache, shape, q, mq)
    compare(o, lse, lens, q, mq, mk, *stored(cache, 1, 128, 200), 0)


def test_nothing_but_itself():
    """a query that shares no group: its own key alone, whose value it returns"""
    lens = [500, 1, 64]
    cache, q, mq, mk, k, v = filled(lens, 16, 4, 2, 128, 4, 1, 2)
    mq.zero_()
    shape = fb.make_shape(4, 2, 500, 128, 4, 1, 0, batch=3)
    o, lse = decode(cache, shape, q, mq)
    ks, vs = stored(cache, 2, 128, 500)
    for b, m in enumerate(lens):
        assert torch.equal(o[b], vs[b, :, m - 1].repeat_interleave(2, 0))
    compare(o, lse, lens, q, mq, mk, ks, vs, 0)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_infinities_and_nan_stay_where_they_are(D):
    """tokens of infinities and NaN that a head does not attend leave it alone, also where another head of its group attends them"""
    lens, Hq = [300], 4
    B, n, K = 1, 300, 4
    g = gen(D)
    shape = fb.make_shape(Hq, 1, n, D, K, 1, 10)
    table, num = table_of(lens, 32)
    cache = pool(shape, 32, table, num, lens)
    k, v = (torch.randn((1, 1, n, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    mk = (1 << (torch.arange(n, device="cuda", dtype=torch.int32) % K))[None].to(torch.int32).contiguous()
    bad = [17, 81, 33]
    k[0, 0, 17, 5] = float("nan")                       # group 1
    v[0, 0, 81, 9] = float("inf")                       # group 1
    v[0, 0, 33, D - 1] = float("nan")                   # group 1
    q = torch.randn((1, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    mq = torch.tensor([1, 2, 4, 8], dtype=torch.int32, device="cuda")
    fb.focus_kv4_append(shape, cache, k, v, mk)
    o, lse = decode(cache, shape, q, mq)
    assert o[0, 1].isnan().all() and lse[0, 1].isnan()
    ks, vs = stored(cache, 1, D, n)
    ks[0, 0, bad], vs[0, 0, bad] = 0, 0
    others = [0, 2, 3]
    for h in others:
        compare(o[:, h:h + 1], lse[:, h:h + 1], lens, q[:, h:h + 1], mq[h:h + 1], mk, ks, vs, 10)
    # and with the head alone: the same
    mq[1] = 1
    o2, lse2 = decode(cache, shape, q, mq)
    assert o2.isfinite().all() and torch.equal(o2[0, others], o[0, others])


def test_bad_pages_and_lengths_are_left_out_and_told():
    lens, P, Hq, Hkv, D = [100, 90, 40], 32, 4, 2, 128
    cache, q, mq, mk, k, v = filled(lens, P, Hq, Hkv, D, 4, 2, 11)
    pages, table, dl = cache.tensors
    shape = fb.make_shape(Hq, Hkv, 100, D, 4, 2, 200, batch=3)
    o, lse = decode(cache, shape, q, mq)
    ks, vs = stored(cache, Hkv, D, 100)
    good = table.clone()
    for entry in (-1, cache.num_pages, 2 ** 31 - 1, -2 ** 31):
        table.copy_(good)
        table[1, 1] = entry
        st = status()
        o1, lse1 = decode(cache, shape, q, mq, st=st)
        assert st.tolist() == [1, 1, 1, entry]
        assert torch.equal(o1[[0, 2]], o[[0, 2]])
        # without the page's keys: attention over the others
        rest = torch.cat([torch.arange(32), torch.arange(64, 90)]).cuda()
        for h in range(Hkv):
            hs = slice(2 * h, 2 * h + 2)
            keep = torch.ones((2, len(rest)), dtype=torch.bool, device="cuda")
            ro, rl, pv, size = kp.attend(q[1, hs], ks[1, h, rest], vs[1, h, rest], keep)
            tol_o, tol_l = kp.tolerances(ro, pv, size, rl, 100)
            assert (o1[1, hs].double() - ro).abs().sub(tol_o).max() <= 0 and (lse1[1, hs].double() - rl).abs().sub(tol_l).max() <= 0
        # append and read pass over it too
        before = pages.clone()
        s10 = fb.make_shape(Hq, Hkv, 60, D, 4, 2, 0, batch=3)
        st = status()
        x = torch.zeros((3, Hkv, 60, D), dtype=torch.bfloat16, device="cuda")
        fb.focus_kv4_append(s10, cache, x, x, torch.zeros((3 * Hkv, 60), dtype=torch.int32, device="cuda"), torch.tensor([0, 60, 0], dtype=torch.int32, device="cuda"), st)
        assert st.tolist() == [1, 1, 1, entry]
        assert torch.equal(pages[good[0].long()], before[good[0].long()])
        out = torch.full((3, Hkv, 100, D), 9.0, dtype=torch.bfloat16, device="cuda")
        out2, st = out.clone(), status()
        fb.focus_kv4_read(fb.make_shape(Hq, Hkv, 100, D, 4, 2, 0, batch=3), cache, None, out, out2, None, st)
        assert st.tolist() == [1, 1, 1, entry] and (out[1, :, 32:64] == 9).all() and torch.equal(out[0], ks[0])
        pages.copy_(before)
    table.copy_(good)
    # lengths
    for wrong in (-1, 101, 2 ** 31 - 1):
        dl[2] = wrong
        st = status()
        o1, lse1 = decode(cache, shape, q, mq, st=st)
        assert st.tolist() == [2, 2, wrong, 100]
        assert torch.equal(o1[:2], o[:2]) and (o1[2] == 0).all() and (lse1[2] == -math.inf).all()
    dl[2] = 40
    s5 = fb.make_shape(Hq, Hkv, 5, D, 4, 2, 0, batch=3)
    x = torch.zeros((3, Hkv, 5, D), dtype=torch.bfloat16, device="cuda")
    m = torch.zeros((3 * Hkv, 5), dtype=torch.int32, device="cuda")
    for length, count in ((4, 5), (40, 6), (40, -1), (-1, 0), (129, 5)):
        dl[2] = length
        before, st = pages.clone(), status()
        fb.focus_kv4_append(s5, cache, x, x, m, torch.tensor([0, 0, count], dtype=torch.int32, device="cuda"), st)
        assert st.tolist() == [2, 2, length, count] and torch.equal(pages, before)
    dl[2] = 40
    st = status()
    fb.focus_kv4_read(s5, cache, torch.tensor([0, 0, -1], dtype=torch.int32, device="cuda"), x, x.clone(), None, st)
    assert st.tolist() == [2, 2, 40, -1]


@pytest.mark.parametrize("D,Hkv,P,count", [(128, 8, 64, 40), (64, 1, 16, 1), (256, 3, 32, 17)])
def test_copy_pages(D, Hkv, P, count):
    shape, g = fb.make_shape(Hkv, Hkv, 1, D, 4, 2, 0), gen(count)
    num = 2 * count + 5
    pages = torch.randint(0, 256, (num, fb.focus_kv4_page_bytes(shape, P)), generator=g, device="cuda", dtype=torch.uint8)
    cache = fb.make_kv4(pages, P)
    pick = torch.randperm(num, generator=g, device="cuda").to(torch.int32)
    src, dst = pick[:count].contiguous(), pick[count:2 * count].contiguous()
    src[count // 2:] = src[0].item()                     # a source may be asked for more than once
    want, st = pages.clone(), status()
    want[dst.long()] = pages[src.long()]
    fb.focus_kv4_copy_pages(shape, cache, src, dst, st)
    assert torch.equal(pages, want) and st.tolist() == [0] * 4
    # pairs outside the pool are passed over, a page onto itself is nothing
    for bad, code in (((-1, 0), 3), ((0, num), 3), ((num, 0), 3), ((2 ** 31 - 1, -2 ** 31), 3), ((3, 3), 0)):
        st = status()
        fb.focus_kv4_copy_pages(shape, cache, torch.tensor([bad[0]], dtype=torch.int32, device="cuda"), torch.tensor([bad[1]], dtype=torch.int32, device="cuda"), st)
        assert torch.equal(pages, want) and st.tolist() == ([3, 0, *bad] if code else [0] * 4)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    fb.focus_kv4_copy_pages(shape, cache, none, none)
    assert torch.equal(pages, want)


def test_pages_beyond_4_gigabytes():
    Hq, Hkv, D, P, n = 16, 8, 128, 256, 700
    shape = fb.make_shape(Hq, Hkv, n, D, 4, 2, 50, batch=2)
    size = fb.focus_kv4_page_bytes(shape, P)
    num = (6 << 30) // size
    pages = torch.empty((num, size), dtype=torch.uint8, device="cuda")
    at = torch.tensor([num - 1, 3, num - 2, num // 2, num - 5, num // 2 + 9], dtype=torch.int32, device="cuda").view(2, 3)
    lens = torch.tensor([700, 650], dtype=torch.int32, device="cuda")
    cache = fb.make_kv4(pages, P, at, lens, KS, VS)
    g = gen(4)
    k, v = (torch.randn((2, Hkv, n, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    mk = torch.randint(0, 16, (2 * Hkv, n), generator=g, device="cuda", dtype=torch.int32)
    mq = torch.randint(0, 16, (2 * Hq,), generator=g, device="cuda", dtype=torch.int32)
    q = torch.randn((2, Hq, D), generator=g, device="cuda").to(torch.bfloat16)
    fb.focus_kv4_append(shape, cache, k, v, mk, lens)
    ks, vs = stored(cache, Hkv, D, n)
    assert torch.equal(ks[0].double().cpu(), kp.rounded(k[0], KS)) and torch.equal(vs[1, :, :650].double().cpu(), kp.rounded(v[1, :, :650], VS))
    fb.focus_kv4_copy_pages(shape, cache, at[0].contiguous(), torch.tensor([num - 7, num - 8, num - 9], dtype=torch.int32, device="cuda"))
    at[0] = torch.tensor([num - 7, num - 8, num - 9], dtype=torch.int32, device="cuda")
    o, lse = decode(cache, shape, q, mq)
    compare(o, lse, [700, 650], q, mq, mk, ks, vs, 50)


def test_replay_with_other_lengths_and_two_streams():
    lens, P, Hq, Hkv, D = [400, 300], 64, 8, 2, 128
    cache, q, mq, mk, k, v = filled(lens, P, Hq, Hkv, D, 4, 2, 21)
    dl = cache.tensors[2]
    shape = fb.make_shape(Hq, Hkv, 448, D, 4, 2, 30, batch=2)
    one = fb.make_shape(Hq, Hkv, 1, D, 4, 2, 30, batch=2)
    kn, vn = (torch.randn((2, Hkv, 1, D), generator=gen(5), device="cuda").to(torch.bfloat16) for _ in range(2))
    mn = torch.full((2 * Hkv, 1), 3, dtype=torch.int32, device="cuda")
    ws = torch.empty(fb.focus_kv4_decode_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(2 * Hq, device="cuda")

    def step(stream=None):
        fb.focus_kv4_append(one, cache, kn, vn, mn, None, None, stream)
        fb.focus_kv4_decode_step(shape, cache, q, mq, o, lse, ws, None, stream)
    dl.copy_(torch.tensor([395, 257]))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for new in ([20, 300], [399, 1], [400, 299]):
        dl.copy_(torch.tensor(new))
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        o.zero_(), lse.zero_()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        step(side)
        side.synchronize()
        assert torch.equal(got[0], o) and torch.equal(got[1], lse) and o.isfinite().all()
    # two decode steps at once, each with its own scratch
    other = torch.empty_like(ws)
    want = decode(cache, shape, q, mq)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [(torch.zeros_like(q), torch.zeros(2 * Hq, device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, w, (a, b) in zip(streams, (ws, other), outs):
            fb.focus_kv4_decode_step(shape, cache, q, mq, a, b, w, None, s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b.view(2, Hq), want[1]) for a, b in outs)


def test_refusals_on_the_gpu():
    lens = [10]
    cache, q, mq, mk, k, v = filled(lens, 16, 18, 2, 128, 4, 2, 3)
    with pytest.raises(fb.FocusError) as e:              # nine query heads per KV head
        decode(cache, fb.make_shape(18, 2, 10, 128, 4, 2, 0), q, mq)
    assert e.value.status == -2
    cache, q, mq, mk, k, v = filled(lens, 16, 4, 2, 128, 4, 2, 3)
    shape = fb.make_shape(4, 2, 10, 128, 4, 2, 0)
    with pytest.raises(fb.FocusError) as e:
        decode(cache, shape, q, mq, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -3
    with pytest.raises(AssertionError):                  # pages of another shape
        decode(cache, fb.make_shape(8, 4, 10, 128, 4, 2, 0), torch.cat([q, q], 1), torch.cat([mq, mq]))
    with pytest.raises(AssertionError):
        decode(cache, fb.make_shape(4, 2, 10, 128, 4, 2, 0, batch=2), torch.cat([q, q]), torch.cat([mq, mq]))


def test_a_refused_append_counts_no_tokens():
    B, Hkv, D = 2, 2, 64
    layer = Kv4Cache(B, 4, Hkv, D, 4, 2, 16, max_tokens=64, num_pages=6, page_tokens=16)
    k = torch.randn((B, Hkv, 5, D), device="cuda").to(torch.bfloat16)
    mk = torch.ones((B * Hkv, 5), dtype=torch.int32, device="cuda")
    layer.append(k, k, mk, [5, 3])
    before = layer.pages.clone(), list(layer.refs), [list(p) for p in layer.held], list(layer.tokens), layer.table.clone(), layer.lens.clone()
    for bad in ((k.float(), k, mk), (k, k[:, :1], mk), (k, k, mk[:, :4])):
        with pytest.raises((AssertionError, fb.FocusError)):
            layer.append(*bad)
    assert torch.equal(layer.pages, before[0]) and (layer.refs, layer.held, layer.tokens) == before[1:4]
    assert torch.equal(layer.table, before[4]) and torch.equal(layer.lens, before[5])
    layer.append(k, k, mk)
    assert layer.tokens == [10, 8] and layer.lens.tolist() == [10, 8] and layer.status.tolist() == [0] * 4


def test_a_serving_loop():
    """norm and rotation, groups, append, decode step by step, a fork, a sequence freed, the pool compacted: against attention in 64 bits
    over what was stored"""
    B, Hq, Hkv, D, K, topk, w = 3, 8, 2, 128, 4, 2, 8
    g = gen(77)
    layer = Kv4Cache(B, Hq, Hkv, D, K, topk, w, max_tokens=160, num_pages=24, page_tokens=16, k_scale=0.5)
    rope, freq = fb.make_rope(D), fb.focus_rope_frequencies(D)[0]
    wq, wk = (1 + 0.1 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
    cent = torch.randn((Hkv, K, D), generator=g, device="cuda")
    kept = {b: [] for b in range(B)}                     # what each sequence has stored: (k, v, mk) per token

    def advance(n, counts, live):
        shape = fb.make_shape(Hq, Hkv, n, D, K, topk, w, batch=B)
        qkv = torch.randn((B, n, Hq + 2 * Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
        x = [t.transpose(1, 2) for t in qkv.split([Hq, Hkv, Hkv], 2)]
        q, k = torch.empty((B, Hq, n, D), dtype=torch.bfloat16, device="cuda"), torch.empty((B, Hkv, n, D), dtype=torch.bfloat16, device="cuda")
        pos = torch.tensor([[layer.tokens[b] + t for t in range(n)] for b in range(B)], dtype=torch.int32, device="cuda")
        fb.focus_qk_norm_rope(shape, rope, x[0], x[1], wq, wk, freq, pos, q, k)
        mq, mk = torch.empty((B * Hq, n), dtype=torch.int32, device="cuda"), torch.empty((B * Hkv, n), dtype=torch.int32, device="cuda")
        fb.focus_assign(shape, q, Hq, cent, mq)
        fb.focus_assign(shape, k, Hkv, cent, mk)
        layer.append(k, x[2], mk, counts)
        kr, vr, mv = kp.rounded(k, 0.5), kp.rounded(x[2], 1.0), mk.view(B, Hkv, n).cpu()
        for b in range(B):
            kept[b] += [(kr[b, :, t], vr[b, :, t], mv[b, :, t]) for t in range(counts[b])]
        last = torch.tensor([max(c, 1) - 1 for c in counts], device="cuda")
        ql = q[torch.arange(B, device="cuda"), :, last].contiguous()
        ml = mq.view(B, Hq, n)[torch.arange(B, device="cuda"), :, last].contiguous().flatten()
        o, lse = torch.empty_like(ql), torch.empty(B * Hq, device="cuda")
        layer.decode(ql, ml, o, lse)
        for b in live:
            k64, v64 = (torch.stack([t[i] for t in kept[b]], 1)[None].cuda() for i in (0, 1))
            m64 = torch.stack([t[2] for t in kept[b]], 1).cuda()
            compare(o[b:b + 1], lse.view(B, Hq)[b:b + 1], [len(kept[b])], ql[b:b + 1], ml.view(B, Hq)[b], m64, k64, v64, w)
        return ql, ml, o, lse

    advance(40, [40, 0, 25], [0, 2])
    layer.fork(0, 1)
    kept[1] = list(kept[0])
    for _ in range(3):
        advance(1, [1, 1, 1], [0, 1, 2])
    layer.free(0)
    kept[0] = []
    ql, ml, o, lse = advance(1, [0, 1, 1], [1, 2])
    assert (o[0] == 0).all() and (lse[:Hq] == -math.inf).all()
    used = layer.compact()
    assert max(p for h in layer.held for p in h) < used
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    layer.decode(ql, ml, o2, lse2)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    advance(30, [30, 7, 20], [0, 1, 2])
    # the cached prefix back in bf16, as a prompt's pass would read it
    k, v = (torch.zeros((B, Hkv, 60, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mk = torch.zeros((B * Hkv, 60), dtype=torch.int32, device="cuda")
    layer.read(k, v, mk)
    for b in range(B):
        n = min(60, len(kept[b]))
        assert torch.equal(k[b, :, :n].double().cpu(), torch.stack([t[0] for t in kept[b][:n]], 1))
        assert torch.equal(v[b, :, :n].double().cpu(), torch.stack([t[1] for t in kept[b][:n]], 1))
    assert layer.status.tolist() == [0] * 4
