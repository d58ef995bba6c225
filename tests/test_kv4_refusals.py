"""4-bit cache, norm and rotation: refusals that no device is asked for, with their exact status.  CPU."""
import ctypes

import pytest

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
