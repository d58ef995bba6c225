"""4-bit cache, norm and rotation: what the host refuses, the structs, page sizes, frequencies, and the bookkeeping of pages.  CPU."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200.kv4_cache import Kv4Cache
from tests import kv4_plain as kp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
S = fb.make_shape(8, 4, 100, 128, 4, 2, 16, batch=2)
R = ctypes.byref


def cache(**kw):
    base = dict(pages=4096, table=4096, lens=4096, num_pages=8, page_tokens=64, max_pages=4, k_scale=1.0, v_scale=0.5)
    base.update(kw)
    return fb.focus_kv4(*(base[f] for f, _ in fb.focus_kv4._fields_))


def heads(H=4, n=100, D=128, ptr=4096, **kw):
    return fb.focus_tensor(ptr, kw.get("sb", H * n * D), kw.get("sh", n * D), kw.get("sn", D))


BAD_CACHES = [dict(pages=None), dict(pages=4104), dict(table=None), dict(lens=None), dict(table=4098), dict(num_pages=0), dict(num_pages=1 << 26),
              dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(max_pages=0), dict(k_scale=0.0), dict(k_scale=3.0),
              dict(v_scale=-1.0), dict(v_scale=float("nan")), dict(k_scale=2.0 ** 17), dict(v_scale=2.0 ** -17), dict(v_scale=float("inf"))]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_a_cache_that_cannot_be_is_refused(kw):
    L, t, big = fb.lib(), heads(), 1 << 30
    q = fb.focus_tensor(4096, 8 * 128, 128, 128)
    c = cache(**kw)
    assert L.focus_kv4_append(R(S), R(c), t, t, 4096, None, None, None) == -1
    assert L.focus_kv4_read(R(S), R(c), None, t, t, None, None, None) == -1
    assert L.focus_kv4_decode_step(R(S), R(c), q, 4096, q, 4096, 4096, big, None, None) == -1
    if not {"table", "lens", "max_pages"} & set(kw):
        assert L.focus_kv4_copy_pages(R(S), R(c), 4096, 4096, 1, None, None) == -1
    assert len(L.focus_last_error()) > 0


def test_cache_calls_refuse_what_does_not_fit():
    L, c, t, big = fb.lib(), cache(), heads(), 1 << 30
    bad = [heads(ptr=None), heads(ptr=4104), heads(sn=132), heads(sb=0), heads(sh=0)]
    for x in bad:
        assert L.focus_kv4_append(R(S), R(c), x, t, 4096, None, None, None) == -1
        assert L.focus_kv4_append(R(S), R(c), t, x, 4096, None, None, None) == -1
        assert L.focus_kv4_read(R(S), R(c), None, x, t, None, None, None) == -1
        assert L.focus_kv4_read(R(S), R(c), None, t, x, None, None, None) == -1
    assert L.focus_kv4_append(R(S), R(c), t, t, None, None, None, None) == -1
    assert L.focus_kv4_append(R(S), None, t, t, 4096, None, None, None) == -1
    assert L.focus_kv4_append(R(fb.make_shape(8, 4, 100, 96, 4, 2, 16)), R(c), t, t, 4096, None, None, None) == -2
    wide = fb.make_shape(1, 1, 1 << 21, 128, 4, 2, 16, batch=1 << 10)
    assert L.focus_kv4_copy_pages(R(S), R(c), None, 4096, 1, None, None) == -1
    assert L.focus_kv4_copy_pages(R(S), R(c), 4096, 4096, -1, None, None) == -1
    assert L.focus_kv4_copy_pages(R(S), R(cache(table=None, lens=None, max_pages=0)), None, None, 0, None, None) == 0
    q = fb.focus_tensor(4096, 8 * 128, 128, 128)
    step = lambda s=S, c=c, q=q, mq=4096, o=q, lse=4096, ws=4096, size=big: L.focus_kv4_decode_step(R(s), R(c), q, mq, o, lse, ws, size, None, None)
    for kw in (dict(mq=None), dict(lse=None), dict(ws=None), dict(ws=4104), dict(q=fb.focus_tensor(None, 1, 1, 1)), dict(o=fb.focus_tensor(None, 1, 1, 1)),
               dict(q=fb.focus_tensor(4098, 8 * 128, 128, 128)), dict(q=fb.focus_tensor(4096, 8 * 128, 129, 128)), dict(q=fb.focus_tensor(4096, 0, 128, 128)),
               dict(c=cache(max_pages=1)), dict(o=fb.focus_tensor(4096, 0, 128, 128))):
        assert step(**kw) == -1, kw
    assert step(size=fb.focus_kv4_decode_workspace_bytes(S) - 1) == -3
    # what the kernels do not take: nine heads a group, too many sequences, a pool of 32 GiB, too many keys in all
    assert step(s=fb.make_shape(36, 4, 100, 128, 4, 2, 16, batch=2)) == -2 and step(s=fb.make_shape(8, 4, 100, 128, 4, 2, 16, batch=1025)) == -2
    P256 = 4 * 256 * (128 + 16 + 4)
    assert step(c=cache(page_tokens=256, num_pages=(1 << 35) // P256 + 1)) == -2
    assert step(s=fb.make_shape(8, 8, 1 << 24, 128, 4, 2, 16, batch=1024), c=cache(max_pages=1 << 18)) == -2
    if not torch.cuda.is_available():
        assert step() in (-4, -5) and L.focus_kv4_append(R(wide), R(c), t, t, 4096, None, None, None) in (-1, -2, -4, -5)


def test_norm_and_rotation_refuse_what_does_not_fit():
    L, q, k = fb.lib(), heads(8), heads(4)
    ok = fb.make_rope(128)
    call = lambda s=S, r=ok, q=q, k=k, wq=4096, wk=4096, f=4096, p=None, qo=q, ko=k: L.focus_qk_norm_rope(R(s), R(r) if r else None, q, k, wq, wk, f, p, qo, ko, None)
    back = lambda s=S, r=ok, q=q, k=k, wq=4096, wk=4096, f=4096, p=None, g=q, gk=k, dq=q, dk=k, dwq=8192, dwk=12288, ws=4096, size=1 << 30: \
        L.focus_qk_norm_rope_bwd(R(s), R(r) if r else None, q, k, wq, wk, f, p, g, gk, dq, dk, dwq, dwk, ws, size, None)
    for r in (None, fb.make_rope(127), fb.make_rope(130), fb.make_rope(-2), fb.focus_rope(128, 2, 1.0, 1e-6), fb.make_rope(128, eps=-1.0),
              fb.make_rope(128, eps=float("nan")), fb.make_rope(128, amplitude=float("inf"))):
        assert call(r=r) == -1 and back(r=r) == -1
    for kw in (dict(f=None), dict(f=4100), dict(wq=4098), dict(wk=4097), dict(p=4098), dict(q=heads(8, ptr=4104)), dict(k=heads(4, sn=132)),
               dict(q=heads(8, ptr=None)), dict(k=heads(4, sb=0))):
        assert call(**kw) == -1 and back(**kw) == -1, kw
    assert call(qo=heads(8, ptr=4104)) == -1 and call(ko=heads(4, ptr=None)) == -1
    for kw in (dict(g=heads(8, ptr=None)), dict(gk=heads(4, ptr=4104)), dict(dq=heads(8, sn=4)), dict(dk=heads(4, ptr=None)), dict(dwq=None), dict(dwk=None),
               dict(wq=None), dict(wk=None), dict(dwq=8194), dict(dwk=8192), dict(ws=None), dict(ws=4104)):
        assert back(**kw) == -1, kw
    assert back(size=fb.focus_qk_norm_rope_bwd_workspace_bytes(S) - 1) == -3
    assert call(s=fb.make_shape(8, 4, 100, 96, 4, 2, 16)) == -2 and fb.focus_qk_norm_rope_bwd_workspace_bytes(fb.make_shape(8, 4, 100, 96, 4, 2, 16)) == 0


def test_structs_match_the_header(tmp_path):
    structs = {"focus_rope": fb.focus_rope, "focus_kv4": fb.focus_kv4}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "focus.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    seen = dict(l.split() for l in subprocess.check_output([str(exe)], text=True).splitlines())
    for name, cls in structs.items():
        assert int(seen[name]) == ctypes.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(seen[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


def test_sizes():
    for D in (64, 128, 256):
        s = fb.make_shape(8, 4, 100, D, 4, 2, 16)
        assert [fb.focus_kv4_page_bytes(s, P) for P in (16, 64, 256)] == [4 * P * (D + D // 8 + 4) for P in (16, 64, 256)]
        assert [fb.focus_kv4_page_bytes(s, P) for P in (0, 8, 24, 512, -16)] == [0] * 5
        # decode scratch: the same for every length, growing with the batch
        w = [fb.focus_kv4_decode_workspace_bytes(fb.make_shape(8, 4, n, D, 4, 2, 16, batch=3)) for n in (1, 100, 1 << 20)]
        assert w[0] == w[1] == w[2] > 0
        w = [fb.focus_kv4_decode_workspace_bytes(fb.make_shape(8, 4, 9, D, 4, 2, 16, batch=b)) for b in range(1, 50)]
        assert w == sorted(w)


def test_frequencies():
    def call(*a, **kw):
        f, amp = fb.focus_rope_frequencies(*a, device="cpu", **kw)
        return f.tolist(), amp
    plain = [10000.0 ** (-2 * i / 64) for i in range(32)]
    close = lambda a, b: all(abs(x - y) <= 1e-14 * abs(y) for x, y in zip(a, b)) and len(a) == len(b)
    f, amp = call(64)
    assert close(f, plain) and amp == 1.0 and f[0] == 1.0
    assert close(call(64, scaling=fb.FOCUS_ROPE_LINEAR, factor=8.0)[0], [x / 8 for x in plain])
    base = 10000.0 * 8 ** (64 / 62)
    f = call(64, scaling=fb.FOCUS_ROPE_BASE, factor=8.0)[0]
    assert close(f, [base ** (-2 * i / 64) for i in range(32)]) and abs(f[-1] * 8 / plain[-1] - 1) < 1e-12       # the slowest pair is slowed by `factor`
    f, amp = call(64, scaling=fb.FOCUS_ROPE_PARTS, factor=8.0, low=1.0, high=32.0, trained=4096)
    turns = [4096 * x / (2 * math.pi) for x in plain]
    assert abs(amp - (0.1 * math.log(8) + 1)) < 1e-6
    for x, t, y in zip(plain, turns, f):
        keep = min(1.0, max(0.0, (t - 1) / 31))
        assert abs(y - (keep * x + (1 - keep) * x / 8)) <= 1e-14 * x
    assert f[0] == plain[0] and abs(f[-1] * 8 / plain[-1] - 1) < 1e-12
    assert call(0)[0] == [] and call(2, scaling=fb.FOCUS_ROPE_BASE, factor=4.0)[0] == [1.0]
    for a, kw in (((-2,), {}), ((3,), {}), ((258,), {}), ((64, 0.0), {}), ((64, float("nan")), {}), ((64,), dict(scaling=4)), ((64,), dict(scaling=1, factor=0.0)),
                  ((64,), dict(scaling=3, factor=2.0, low=4.0, high=4.0)), ((64,), dict(scaling=3, factor=2.0, trained=0.0))):
        with pytest.raises(fb.FocusError) as e:
            fb.focus_rope_frequencies(*a, device="cpu", **kw)
        assert e.value.status == -1


def test_plain_form_of_the_codes():
    """the 64-bit form that the GPU is held to, on cases by hand"""
    x = torch.zeros(16)
    x[:8] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    x[8:12] = torch.tensor([-0.26, -5.01, 0.1, -0.1])
    c, s = kp.quantise(x, 1.0)
    assert kp.SCALES[s].tolist() == [1.0] and c.tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 9, 15, 0, 8, 0, 0, 0, 0]
    assert kp.quantise(torch.full((16,), 1e30), 1.0)[1].item() == 126 and kp.rounded(torch.full((16,), -1e30), 0.5).tolist() == [-1344.0] * 16
    assert kp.rounded(torch.full((16,), 2.0 ** -8), 1.0).abs().max() == 0.0           # a scale of 2^-8 / 6 is below half of the smallest


def bookkeeping(pages=8, sequences=3, P=16, most=64):
    c = Kv4Cache(sequences, 4, 2, 64, 4, 2, 16, most, pages, P, device="cpu")
    c._push = lambda stream=None: None
    c.moved = []
    c._move = lambda pairs, stream=None: c.moved.extend(pairs)
    return c


def consistent(c):
    count = [0] * len(c.refs)
    for b, pages in enumerate(c.held):
        assert len(pages) == -(-c.tokens[b] // c.P) and len(set(pages)) == len(pages)
        for p in pages:
            count[p] += 1
    assert count == c.refs


def test_pages_of_a_pool():
    c = bookkeeping()
    c.reserve([20, 0, 16])
    assert c.held == [[0, 1], [], [2]] and c.tokens == [20, 0, 16] and c.moved == []
    c.fork(0, 1)
    assert c.held[1] == [0, 1] and c.refs[:3] == [2, 2, 1]
    consistent(c)
    c.reserve([1, 0, 0])                       # writes to page 1, which sequence 1 shares: copied
    assert c.moved == [(1, 3)] and c.held[0] == [0, 3] and c.held[1] == [0, 1]
    c.reserve([0, 1, 0])                       # its own by now
    assert c.moved == [(1, 3)]
    c.reserve([0, 0, 1])                       # the last page is full: a new one, none copied
    assert c.held[2] == [2, 4] and c.moved == [(1, 3)]
    consistent(c)
    c.free(1)
    assert c.refs[1] == 0 and c.refs[0] == 1
    consistent(c)
    c.moved.clear()
    assert c.compact() == 4 and c.moved == [(4, 1)] and c.held == [[0, 3], [], [2, 1]]
    consistent(c)
    assert c.compact() == 4 and c.moved == [(4, 1)]


def test_a_pool_that_is_used_up_changes_nothing():
    c = bookkeeping(pages=4)
    c.reserve([16, 16, 20])
    before = (list(c.refs), [list(h) for h in c.held], list(c.tokens))
    for counts, status in (([1, 0, 0], -3), ([0, 0, 45], -3), ([0, 0], -1), ([0, -1, 0], -1)):
        with pytest.raises(fb.FocusError) as e:
            c.reserve(counts)
        assert e.value.status == status and (c.refs, c.held, c.tokens) == before
    with pytest.raises(fb.FocusError):
        c.fork(0, 1)
    with pytest.raises(fb.FocusError):
        c.fork(0, 0)
    c.free(0)
    c.fork(2, 0)
    with pytest.raises(fb.FocusError):         # one page is free: the first to write takes it for its copy, and two are wanted
        c.reserve([13, 0, 13])
    assert c.tokens == [20, 16, 20] and c.moved == []
    c.reserve([1, 0, 1])                       # the other keeps the page, which is its own then
    assert c.moved == [(3, 0)]
    consistent(c)


def test_forks_of_forks_and_random_use():
    g = torch.Generator().manual_seed(1)
    c = bookkeeping(pages=24, sequences=6, most=80)
    draw = lambda m: int(torch.randint(0, m, (1,), generator=g))
    for _ in range(400):
        what = draw(4)
        try:
            if what == 0:
                c.reserve([draw(20) if draw(2) else 0 for _ in range(6)])
            elif what == 1:
                c.fork(draw(6), draw(6))
            elif what == 2:
                c.free(draw(6))
            else:
                c.compact()
                assert all(r == 0 for r in c.refs[sum(r > 0 for r in c.refs):])
        except fb.FocusError:
            pass
        consistent(c)
