"""Shapes that the attention's backward passes refuse: their workspace queries say so too, before anything is built around them (no GPU needed)."""
import pytest

from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200.gate_layer import GateLayer
from test_bwd_refusals import attn_args, shape

BOTH = [dict(batch=20000), dict(scale=float("inf")), dict(scale=2.0 ** -101), dict(n=1 << 30, Hq=512, Hkv=512), dict(n=0), dict(D=96)]
GATE = [dict(softcap=5.0), dict(D=256, K=17, topk=1), dict(D=256, K=32, topk=1)]


@pytest.mark.parametrize("kw", BOTH + GATE)
def test_no_size_for_what_is_refused(kw):
    s = shape(**kw)
    for gate in (False, True) if kw in BOTH else (True,):
        assert (fb.focus_gate_attn_bwd_workspace_bytes if gate else fb.focus_attn_bwd_workspace_bytes)(s) == 0
        assert fb.lib().focus_last_error()
        assert attn_args(s, gate) in (-1, -2)
    if kw in GATE:
        assert fb.focus_attn_bwd_workspace_bytes(s) > 0


def test_sizes_of_what_is_taken():
    for kw in (dict(), dict(D=256, K=16), dict(K=32), dict(batch=16383), dict(scale=2.0 ** -100), dict(n=1 << 20)):
        s = shape(**kw)
        assert 0 < fb.focus_attn_bwd_workspace_bytes(s) and 0 < fb.focus_gate_attn_bwd_workspace_bytes(s)
        # (the size is what the call asks for)
        assert attn_args(s, False, size=fb.focus_attn_bwd_workspace_bytes(s) - 1) == -3 and attn_args(s, True, size=fb.focus_gate_attn_bwd_workspace_bytes(s) - 1) == -3


@pytest.mark.parametrize("bad", [dict(D=256, K=17), dict(batch=20000), dict(scale=2.0 ** -101)])
def test_no_layer_of_a_shape_that_only_the_backward_pass_refuses(bad):
    with pytest.raises(fb.FocusError, match="K = 17|65535|2\\^-100"):
        GateLayer(**{**dict(batch=1, Hq=4, Hkv=2, n=10, D=64, K=4, d_model=64, d_g=16, window=0, lam=1.0), **bad})


@pytest.mark.parametrize("lam", [3e38, -3e38, 2.0 ** 101])
def test_slopes_whose_products_are_no_numbers(lam):
    """lambda log2(e) is infinite from 2.4e38 on, and times an assignment of 0 nothing at all"""
    assert attn_args(shape(), True, lam=lam) == -2 and "lambda" in fb.lib().focus_last_error().decode()
    assert attn_args(shape(), True, lam=2.0 ** 100, size=1000) == -3
