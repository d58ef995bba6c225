"""4-bit cache, norm and rotation: refusals that no device is asked for, with their exact status.  CPU."""
import ctypes
import math
import types

import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from tests.test_kv4_host import cache, heads

R = ctypes.byref


def decode(shape, c=None, mq=4096, lse=4096, o=4096, status=None):
    vec = lambda p: fb.focus_tensor(p, 8 * 128, 128, 128)
    return fb.lib().focus_kv4_decode_step(R(shape), R(c or cache()), vec(4096), mq, vec(o), lse, 4096, 1 << 30, status, None)


def decode_shape(**kw):
    a = dict(Hq=8, Hkv=4, n=100, D=128, K=4, topk=2, window=16, batch=2)
    a.update(kw)
    return fb.make_shape(**a)


@pytest.mark.parametrize("kw", [dict(scale=float("inf")), dict(softcap=float("inf")), dict(scale=float("nan")), dict(softcap=float("nan"))])
def test_scales_and_caps_that_are_no_numbers(kw):
    assert decode(decode_shape(**kw)) == -1


BIG = 1 << 31


def append(shape, c=None, k=None, v=None, mk=4096, counts=None, status=None):
    t = heads(shape.Hkv, shape.n)
    return fb.lib().focus_kv4_append(R(shape), R(c or cache()), k or t, v or t, mk, counts, status, None)


def read(shape, c=None, first=None, mk=None, status=None):
    t = heads(shape.Hkv, shape.n)
    return fb.lib().focus_kv4_read(R(shape), R(c or cache()), first, t, t, mk, status, None)


def copy(count, c=None, src=4096, dst=4096, status=None):
    return fb.lib().focus_kv4_copy_pages(R(decode_shape()), R(c or cache()), src, dst, count, status, None)


def asked(rc):
    """all that the host can check has been passed: it is the device that is missing here (or one of another kind)"""
    if torch.cuda.is_available():
        pytest.skip("would be launched")
    return rc in (-4, -5)


@pytest.mark.parametrize("batch,Hkv,n", [(1 << 10, 1, 1 << 21), (2, 1, 1 << 30), (1 << 15, 4, 1 << 14), (3, 7, 102261127)])
def test_rows_of_an_append_or_a_read(batch, Hkv, n):
    """batch * Hkv * n is below 2^31"""
    assert batch * Hkv * n >= BIG and batch * Hkv * (n - 1) < BIG
    at = decode_shape(Hq=Hkv, Hkv=Hkv, n=n, batch=batch)
    assert append(at) == -2 and read(at) == -2
    below = decode_shape(Hq=Hkv, Hkv=Hkv, n=n - 1, batch=batch)
    assert asked(append(below)) and asked(read(below))


def test_pages_of_a_copy():
    """16 KB of a page are a CTA's, of which there are fewer than 2^31"""
    chunks = -(-(4 * 256 * (128 + 16 + 4) // 16) // 1024)
    most = (BIG - 1) // chunks
    c = cache(page_tokens=256)
    assert copy(most + 1, c) == -2 and asked(copy(most, c))


def rope(shape, back=False, rotary=128):
    L, q, k = fb.lib(), heads(shape.Hq, shape.n), heads(shape.Hkv, shape.n)
    r = fb.make_rope(rotary)
    if not back:
        return L.focus_qk_norm_rope(R(shape), R(r), q, k, 4096, 4096, 4096, None, q, k, None)
    return L.focus_qk_norm_rope_bwd(R(shape), R(r), q, k, 4096, 4096, 4096, None, q, k, q, k, 8192, 12288, 4096, BIG, None)


@pytest.mark.parametrize("rotary", [128, 70])
def test_tokens_of_norm_and_rotation(rotary):
    """batch * n is below 2^30, and the passes over all heads below 2^31 (backward)"""
    for batch, n in ((1, 1 << 30), (1 << 10, 1 << 20), (3, 357913942)):
        at, below = (decode_shape(Hq=1, Hkv=1, n=m, batch=batch) for m in (n, n - 1))
        for back in (False, True):
            assert rope(at, back, rotary) == -2 and asked(rope(below, back, rotary))
    many = decode_shape(Hq=1 << 10, Hkv=1, n=(1 << 30) - 1, batch=1)
    assert asked(rope(many, False, rotary))
    assert rope(many, True, rotary) == -2 if rotary == 128 else asked(rope(many, True, rotary))
    if rotary == 128:                        # 1024 heads of a token are 32 passes
        many = [decode_shape(Hq=1 << 10, Hkv=1, n=m, batch=1) for m in (1 << 26, (1 << 26) - 1)]
        assert rope(many[0], True) == -2 and asked(rope(many[1], True))


@pytest.mark.parametrize("off", [1, 2, 3])
def test_misaligned_words(off):
    """masks, counts, lists, log-sum-exps and the status are read and written four bytes at a time"""
    s, p = decode_shape(), 4096 + off
    one = decode_shape(n=100)
    for kw in (dict(mk=p), dict(counts=p), dict(status=p)):
        assert append(one, **kw) == -1, kw
    for kw in (dict(first=p), dict(mk=p), dict(status=p)):
        assert read(one, **kw) == -1, kw
    for kw in (dict(src=p), dict(dst=p), dict(status=p)):
        assert copy(3, **kw) == -1, kw
    for kw in (dict(mq=p), dict(lse=p), dict(status=p), *([dict(o=p)] if off % 2 else [])):
        assert decode(s, **kw) == -1, kw
    if off == 2:
        assert asked(decode(s, o=p))         # (o is written number by number)


class OnGpu:
    """a tensor as far as the binding looks at one, for calls whose pointers nobody follows"""
    def __init__(self, dtype, *shape, cuda=True, contiguous=True):
        self.dtype, self.shape, self.is_cuda, self.flat = dtype, shape, cuda, contiguous

    def stride(self):
        return tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def is_contiguous(self):
        return self.flat

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 4096


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched")
@pytest.mark.parametrize("kw,error", [(dict(), fb.FocusError), (dict(cuda=False), AssertionError), (dict(contiguous=False), AssertionError)])
def test_scratch_that_is_not_on_the_gpu_or_not_in_one_piece(monkeypatch, kw, error):
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    stream = types.SimpleNamespace(cuda_stream=0)
    s = decode_shape()
    ws = OnGpu(torch.uint8, 1 << 30, **kw)
    c = cache()
    c.tensors = OnGpu(torch.uint8, 8, fb.focus_kv4_page_bytes(s, 64)), OnGpu(i32, 2, 4), OnGpu(i32, 2)
    vec = OnGpu(bf, 2, 8, 128)
    with pytest.raises(error):
        fb.focus_kv4_decode_step(s, c, vec, OnGpu(i32, 16), vec, OnGpu(f32, 16), ws, None, stream)
    q, k, w = OnGpu(bf, 2, 8, 100, 128), OnGpu(bf, 2, 4, 100, 128), OnGpu(f32, 128)
    other = OnGpu(f32, 128)
    monkeypatch.setattr(other, "data_ptr", lambda: 8192, raising=False)
    with pytest.raises(error):
        fb.focus_qk_norm_rope_bwd(s, fb.make_rope(128), q, k, w, w, OnGpu(torch.float64, 64), None, q, k, q, k, w, other, ws, stream)
