"""What the backward entry points refuse on the host, before the device is asked (no GPU needed)."""
import ctypes as C

import pytest

from paper_2604_03260_b200 import binding as fb

A = 1 << 20        # an address that nothing looks at


def shape(**kw):
    base = dict(Hq=4, Hkv=2, n=300, D=128, K=4, topk=2, window=16)
    base.update(kw)
    return fb.make_shape(**base)


def heads(s, H, at, dn=0):
    return fb.focus_tensor(at, H * s.n * s.D, s.n * s.D, s.D + dn)


def attn_args(s, gate, **kw):
    a = dict(q=heads(s, s.Hq, A), k=heads(s, s.Hkv, 2 * A), v=heads(s, s.Hkv, 3 * A), mq=None, mk=None, tiles=None, layout=0, g=9 * A, lam=10.0, o=heads(s, s.Hq, 4 * A), lse=5 * A,
             do=heads(s, s.Hq, 6 * A), dq=heads(s, s.Hq, 7 * A), dk=heads(s, s.Hkv, 8 * A), dv=heads(s, s.Hkv, 10 * A), dg=11 * A, ws=12 * A, size=1 << 40, status=None)
    a.update(kw)
    L = fb.lib()
    tail = [a["ws"], a["size"], a["status"], None]
    if gate:
        return L.focus_gate_attn_bwd(C.byref(s), a["q"], a["k"], a["v"], a["g"], a["lam"], a["o"], a["lse"], a["do"], a["dq"], a["dk"], a["dv"], a["dg"], *tail)
    return L.focus_attn_bwd(C.byref(s), a["q"], a["k"], a["v"], a["mq"], a["mk"], a["tiles"], a["layout"], a["o"], a["lse"], a["do"], a["dq"], a["dk"], a["dv"], *tail)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("bad,status", [
    (lambda s: dict(q=fb.focus_tensor(None, 1, 1, 1)), -1), (lambda s: dict(k=heads(s, s.Hkv, A + 8)), -1), (lambda s: dict(do=heads(s, s.Hq, A, 4)), -1),
    (lambda s: dict(dv=heads(s, s.Hkv, A + 2)), -1), (lambda s: dict(lse=None), -1), (lambda s: dict(lse=A + 2), -1), (lambda s: dict(ws=None), -1), (lambda s: dict(ws=A + 8), -1),
    (lambda s: dict(size=1000), -3), (lambda s: dict(dq=heads(s, s.Hq, A)), -1), (lambda s: dict(dk=heads(s, s.Hkv, 3 * A)), -1), (lambda s: dict(dk=heads(s, s.Hkv, 10 * A)), -1),
    (lambda s: dict(status=A + 1), -1),
])
def test_attention(gate, bad, status):
    s = shape()
    assert attn_args(s, gate, **bad(s)) == status and fb.lib().focus_last_error()


@pytest.mark.parametrize("kw,status", [(dict(Hq=3), -1), (dict(D=96), -2), (dict(n=0), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(batch=70000), -2)])
def test_attention_shapes(kw, status):
    s = shape(**kw)
    for gate in (False, True):
        big = dict(q=fb.focus_tensor(A, 8, 8, 128)) if "batch" in kw else {}
        assert attn_args(s, gate, **big) == status


def test_masks_and_gate():
    s = shape()
    assert attn_args(s, False, tiles=A) == -1 and attn_args(s, False, tiles=A, mq=A, mk=A + 2) == -1 and attn_args(s, False, tiles=A + 16, mq=A, mk=A) == -1
    assert attn_args(s, False, tiles=A, mq=A, mk=A, layout=9) == -1
    assert attn_args(s, True, g=None) == -1 and attn_args(s, True, dg=None) == -1 and attn_args(s, True, g=A + 4) == -1 and attn_args(s, True, dg=9 * A) == -1
    assert attn_args(s, True, lam=float("nan")) == -1 and attn_args(shape(softcap=5.0), True) == -2 and attn_args(shape(D=256, K=17, topk=1), True) == -2
    assert fb.focus_attn_bwd_workspace_bytes(shape(n=0)) == 0 and fb.focus_gate_attn_bwd_workspace_bytes(s) > fb.focus_attn_bwd_workspace_bytes(s) > 0


def router_args(s, **kw):
    a = dict(h=A, sb=300 * 64, sn=64, d=64, dg=16, Wg=2 * A, C=3 * A, ds=4 * A, dh=5 * A, db=300 * 64, dn=64, dWg=6 * A, dC=7 * A, ws=8 * A, size=1 << 40)
    a.update(kw)
    return fb.lib().focus_router_scores_bwd(C.byref(s), *a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(h=None), -1), (dict(h=A + 8), -1), (dict(d=60), -1), (dict(d=0), -1), (dict(dg=0), -1), (dict(sn=60), -1), (dict(sn=68), -1), (dict(dn=56), -1), (dict(ds=A + 4), -1), (dict(Wg=A + 2), -1),
    (dict(dWg=None), -1), (dict(dWg=2 * A), -1), (dict(dC=6 * A), -1), (dict(ws=A + 4), -1), (dict(size=16), -3), (dict(dh=A, dn=72), -1), (dict(d=1 << 21, sn=1 << 21, dn=1 << 21), -2),
])
def test_router(kw, status):
    assert router_args(shape(), **kw) == status and fb.lib().focus_last_error()


def test_router_workspace():
    assert fb.focus_router_scores_bwd_workspace_bytes(shape(), 60, 16) == 0 and fb.focus_router_scores_bwd_workspace_bytes(shape(), 64, 16) > 0
    assert router_args(shape(batch=2), sb=0) == -1 and router_args(shape(batch=2), db=0) == -1


def clip(entries, count=None, bound=1.0, norm=None, ws=A, size=1 << 20):
    g = (fb.focus_grad * max(1, len(entries)))(*[fb.focus_grad(*e) for e in entries])
    return fb.lib().focus_grad_clip(g, len(entries) if count is None else count, bound, norm, ws, size, None)


@pytest.mark.parametrize("entry,status", [((None, A, 5, 0), -1), ((A, None, 5, 0), -1), ((A, A, -1, 0), -1), ((A, A, 5, 2), -1), ((A + 2, A + 2, 5, 0), -1), ((A, A + 1, 5, 1), -1), ((A, A, 1 << 41, 0), -2)])
def test_clip_entries(entry, status):
    assert clip([(A, A, 4, 0), entry]) == status


def test_clip():
    assert clip([], count=-1) == -1 and fb.lib().focus_grad_clip(None, 3, 1.0, None, A, 1 << 20, None) == -1
    assert clip([], bound=-1.0) == -1 and clip([], bound=float("nan")) == -1 and clip([], norm=A + 2) == -1 and clip([], ws=None) == -1 and clip([], ws=A + 8) == -1 and clip([], size=8) == -3


def test_scales_that_lse_cannot_be_divided_by():
    assert attn_args(shape(scale=2.0 ** -101), False) == -2 and attn_args(shape(scale=2.0 ** -101), True) == -2
    assert attn_args(shape(scale=2.0 ** -100), False, size=1000) == -3


def test_layer_of_a_shape_that_is_refused():
    from paper_2604_03260_b200.gate_layer import GateLayer
    for bad in (dict(Hq=3), dict(D=96), dict(d_model=60), dict(K=40)):
        with pytest.raises(fb.FocusError):
            GateLayer(**{**dict(batch=1, Hq=4, Hkv=2, n=10, D=64, K=4, d_model=64, d_g=16, window=0, lam=1.0), **bad})
