"""Binding of libfocus_b200.so: same names as the C ABI (include/focus.h), argument marshalling only, through ctypes; the
calls of a decode step and of a short prompt take the same arguments through csrc/marshal.cpp where that is built for this torch.
torch supplies device memory and the current stream; every step of the path runs inside the library's CUDA kernels.  There is no CPU
fallback: loading fails loudly when the library has not been built (``python -m paper_2604_03260_b200.build``)."""
from __future__ import annotations

import ctypes as C
import math
import os
import warnings

import torch

from . import build as _build

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfocus_b200.so")

FOCUS_LAYOUT_ORIGINAL = 0
FOCUS_LAYOUT_CLASS_SORTED = 1
FOCUS_LAYOUT_AUTO = 2
FOCUS_LAYOUT_SORTED_LOCAL = 3
FOCUS_LAYOUT_GROUP_MAJOR = 4
FOCUS_MAX_CLASSES = 64
FOCUS_ROPE_PLAIN = 0
FOCUS_ROPE_LINEAR = 1
FOCUS_ROPE_BASE = 2
FOCUS_ROPE_PARTS = 3


class focus_shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("n", C.c_int32), ("D", C.c_int32),
                ("K", C.c_int32), ("topk", C.c_int32), ("window", C.c_int32), ("scale", C.c_float),
                ("softcap", C.c_float)]


class focus_tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64)]


class focus_tiles_layout(C.Structure):
    _fields_ = [("layout", C.c_int32), ("nqt", C.c_int32), ("nkt", C.c_int32), ("nkw", C.c_int32),
                ("total_bytes", C.c_size_t), ("counters", C.c_size_t),
                ("orq", C.c_size_t), ("andq", C.c_size_t), ("ork", C.c_size_t), ("andk", C.c_size_t),
                ("gbits", C.c_size_t), ("live", C.c_size_t), ("live_cnt", C.c_size_t),
                ("kany", C.c_size_t), ("kall", C.c_size_t),
                ("nqp", C.c_int32), ("nkp", C.c_int32),
                ("ncls_q", C.c_size_t), ("ncls_k", C.c_size_t), ("cls_q", C.c_size_t), ("cls_k", C.c_size_t),
                ("cnt_q", C.c_size_t), ("cnt_k", C.c_size_t),
                ("seg_q", C.c_size_t), ("seg_k", C.c_size_t), ("perm_q", C.c_size_t), ("perm_k", C.c_size_t),
                ("qrange", C.c_size_t), ("order", C.c_size_t), ("gbits_s", C.c_size_t), ("qs", C.c_size_t), ("ks", C.c_size_t),
                ("vs", C.c_size_t), ("scratch", C.c_size_t), ("o_sorted", C.c_size_t), ("o_local", C.c_size_t),
                ("lse_local", C.c_size_t)]


class focus_rope(C.Structure):
    _fields_ = [("rotary", C.c_int32), ("interleaved", C.c_int32), ("amplitude", C.c_float), ("eps", C.c_float)]


class focus_kv4(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("table", C.c_void_p), ("lens", C.c_void_p), ("num_pages", C.c_int32), ("page_tokens", C.c_int32),
                ("max_pages", C.c_int32), ("k_scale", C.c_float), ("v_scale", C.c_float)]


class focus_grad(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("count", C.c_int64), ("dtype", C.c_int32)]


class focus_grads(C.Structure):
    """a list of gradients (make_grad_list), which holds their tensors"""
    _fields_ = [("grads", C.c_void_p), ("count", C.c_int32)]


class FocusError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"focus status {status}: {message}")
        self.status = status


_lib = None
_marshal = None         # csrc/marshal.cpp


def lib():
    global _lib, _marshal
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2604_03260_b200.build` "
                              "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        SP = C.POINTER(focus_shape)
        L.focus_version.restype = C.c_int
        L.focus_status_string.restype = C.c_char_p
        L.focus_status_string.argtypes = [C.c_int]
        L.focus_last_error.restype = C.c_char_p
        L.focus_assign.restype = C.c_int
        L.focus_assign.argtypes = [SP, focus_tensor, i32, vp, vp, vp, f32, vp]
        L.focus_assign_hidden.restype = C.c_int
        L.focus_assign_hidden.argtypes = [SP, vp, C.c_int64, C.c_int64, i32, i32, vp, vp, vp, vp, vp, vp, vp, f32, vp]
        L.focus_tiles_layout_of.restype = C.c_int
        L.focus_tiles_layout_of.argtypes = [SP, i32, C.POINTER(focus_tiles_layout)]
        L.focus_tiles_workspace_bytes.restype = sz
        L.focus_tiles_workspace_bytes.argtypes = [SP, i32]
        L.focus_build_tiles.restype = C.c_int
        L.focus_build_tiles.argtypes = [SP, vp, vp, i32, vp, sz, vp]
        L.focus_attn_fwd.restype = C.c_int
        L.focus_attn_fwd.argtypes = [SP, focus_tensor, focus_tensor, focus_tensor, vp, vp, vp, i32, focus_tensor, vp,
                                     vp, vp]
        L.focus_decode_workspace_bytes.restype = sz
        L.focus_decode_workspace_bytes.argtypes = [SP]
        L.focus_decode_step.restype = C.c_int
        L.focus_decode_step.argtypes = [SP, focus_tensor, focus_tensor, focus_tensor, vp, vp, focus_tensor, vp, vp, sz, vp]
        L.focus_router_scores.restype = C.c_int
        L.focus_router_scores.argtypes = [SP, vp, C.c_int64, C.c_int64, i32, i32, vp, vp, vp, vp, vp]
        L.focus_soft_ld.restype = i32
        L.focus_soft_ld.argtypes = [i32]
        L.focus_sinkhorn_workspace_bytes.restype = sz
        L.focus_sinkhorn_workspace_bytes.argtypes = [SP, i32]
        L.focus_sinkhorn.restype = C.c_int
        L.focus_sinkhorn.argtypes = [SP, vp, f32, i32, vp, sz, vp, vp]
        L.focus_sinkhorn_bwd_workspace_bytes.restype = sz
        L.focus_sinkhorn_bwd_workspace_bytes.argtypes = [SP, i32]
        L.focus_sinkhorn_bwd.restype = C.c_int
        L.focus_sinkhorn_bwd.argtypes = [SP, vp, f32, i32, vp, sz, vp, vp, vp]
        L.focus_gate_attn_fwd.restype = C.c_int
        L.focus_gate_attn_fwd.argtypes = [SP, focus_tensor, focus_tensor, focus_tensor, vp, f32, focus_tensor, vp, vp, vp]
        RP, KP, ft = C.POINTER(focus_rope), C.POINTER(focus_kv4), focus_tensor
        f64 = C.c_double
        L.focus_rope_frequencies.restype = C.c_int
        L.focus_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp, C.POINTER(f32)]
        L.focus_qk_norm_rope.restype = C.c_int
        L.focus_qk_norm_rope.argtypes = [SP, RP, ft, ft, vp, vp, vp, vp, ft, ft, vp]
        L.focus_qk_norm_rope_bwd_workspace_bytes.restype = sz
        L.focus_qk_norm_rope_bwd_workspace_bytes.argtypes = [SP]
        L.focus_qk_norm_rope_bwd.restype = C.c_int
        L.focus_qk_norm_rope_bwd.argtypes = [SP, RP, ft, ft, vp, vp, vp, vp, ft, ft, ft, ft, vp, vp, vp, sz, vp]
        L.focus_kv4_page_bytes.restype = sz
        L.focus_kv4_page_bytes.argtypes = [SP, i32]
        L.focus_kv4_append.restype = C.c_int
        L.focus_kv4_append.argtypes = [SP, KP, ft, ft, vp, vp, vp, vp]
        L.focus_kv4_read.restype = C.c_int
        L.focus_kv4_read.argtypes = [SP, KP, vp, ft, ft, vp, vp, vp]
        L.focus_kv4_copy_pages.restype = C.c_int
        L.focus_kv4_copy_pages.argtypes = [SP, KP, vp, vp, i32, vp, vp]
        L.focus_kv4_decode_workspace_bytes.restype = sz
        L.focus_kv4_decode_workspace_bytes.argtypes = [SP]
        L.focus_kv4_decode_step.restype = C.c_int
        L.focus_kv4_decode_step.argtypes = [SP, KP, ft, vp, ft, vp, vp, sz, vp, vp]
        L.focus_attn_bwd_workspace_bytes.restype = sz
        L.focus_attn_bwd_workspace_bytes.argtypes = [SP]
        L.focus_attn_bwd.restype = C.c_int
        L.focus_attn_bwd.argtypes = [SP, ft, ft, ft, vp, vp, vp, i32, ft, vp, ft, ft, ft, ft, vp, sz, vp, vp]
        L.focus_gate_attn_bwd_workspace_bytes.restype = sz
        L.focus_gate_attn_bwd_workspace_bytes.argtypes = [SP]
        L.focus_gate_attn_bwd.restype = C.c_int
        L.focus_gate_attn_bwd.argtypes = [SP, ft, ft, ft, vp, f32, ft, vp, ft, ft, ft, ft, vp, vp, sz, vp, vp]
        L.focus_router_scores_bwd_workspace_bytes.restype = sz
        L.focus_router_scores_bwd_workspace_bytes.argtypes = [SP, i32, i32]
        L.focus_router_scores_bwd.restype = C.c_int
        L.focus_router_scores_bwd.argtypes = [SP, vp, C.c_int64, C.c_int64, i32, i32, vp, vp, vp, vp, C.c_int64, C.c_int64, vp, vp, vp, sz, vp]
        L.focus_grad_clip_workspace_bytes.restype = sz
        L.focus_grad_clip_workspace_bytes.argtypes = []
        L.focus_grad_clip.restype = C.c_int
        L.focus_grad_clip.argtypes = [vp, i32, f32, vp, vp, sz, vp]
        L.focus_count_kept.restype = C.c_int
        L.focus_count_kept.argtypes = [SP, vp, vp, vp, vp]
        L.focus_count_kept_noalloc.restype = C.c_int
        L.focus_count_kept_noalloc.argtypes = [SP, vp, vp, vp, vp]
        L.focus_selftest_umma.restype = C.c_int
        L.focus_selftest_umma.argtypes = [i32, vp, vp, vp, vp, vp, vp, vp, vp]
        L.focus_selftest_umma_pair.restype = C.c_int
        L.focus_selftest_umma_pair.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
        L.focus_selftest_mma_rate.restype = C.c_int
        L.focus_selftest_mma_rate.argtypes = [i32, i32, i32, i32, i32, vp, vp]
        L.focus_selftest_stalled_wait.restype = C.c_int
        L.focus_selftest_stalled_wait.argtypes = [SP, focus_tensor, focus_tensor, focus_tensor, focus_tensor, vp, C.c_uint64, vp, vp]
        L.focus_selftest_stalled_exchange.restype = C.c_int
        L.focus_selftest_stalled_exchange.argtypes = [SP, vp, f32, i32, vp, sz, C.c_int64, i32, vp, vp]
        _marshal, _lib = _load_marshal(L), L
    return _lib


class _Ctypes:
    """in the place of csrc/marshal.cpp where that cannot be loaded: knows no argument, so that every call goes through ctypes"""
    @staticmethod
    def assign(*args):
        return None
    assign_hidden = build_tiles = attn_fwd = decode_step = assign
    attn_bwd = gate_attn_bwd = router_scores_bwd = grad_clip = assign
    qk_norm_rope = qk_norm_rope_bwd = kv4_append = kv4_read = kv4_copy_pages = kv4_decode_step = assign


def _load_marshal(L):
    """csrc/marshal.cpp, if it was built for this torch and this Python: it knows the layout of their objects"""
    try:
        from . import _marshal as m
        if getattr(m, "built_for", None) != _build.marshal_abi():
            raise ImportError(f"{m.__file__} was built for another torch or Python ({getattr(m, 'built_for', None)}, here {_build.marshal_abi()})")
    except ImportError as e:
        warnings.warn(f"{e}: short calls take some 10 us longer through ctypes; `python -m paper_2604_03260_b200.build` builds the module", RuntimeWarning)
        return _Ctypes
    at = lambda *entries: (C.cast(f, C.c_void_p).value for f in entries)
    m.init(focus_shape, *at(L.focus_assign, L.focus_assign_hidden, L.focus_build_tiles, L.focus_attn_fwd, L.focus_decode_step))
    m.init_kv4(focus_rope, focus_kv4, *at(L.focus_qk_norm_rope, L.focus_qk_norm_rope_bwd, L.focus_kv4_append, L.focus_kv4_read, L.focus_kv4_copy_pages,
                                          L.focus_kv4_decode_step))
    m.init_bwd(focus_grads, *at(L.focus_attn_bwd, L.focus_gate_attn_bwd, L.focus_router_scores_bwd, L.focus_grad_clip))
    return m


def _check(rc):
    if rc != 0:
        raise FocusError(rc, lib().focus_last_error().decode())


def _short():
    """The calls whose GPU work is as short as their marshalling.  They answer with a status, or None when an argument is not of
    the usual kind; it then goes the way of the other entry points."""
    if _marshal is None:
        lib()
    return _marshal


# Addresses and stream handles as integers, one look at a tensor's strides, the current stream's handle without a Stream object
# around it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _p(t):
    return t.data_ptr() if t is not None else None


def make_shape(Hq, Hkv, n, D, K, topk, window, scale=0.0, softcap=0.0, batch=1) -> focus_shape:
    return focus_shape(batch, Hq, Hkv, n, D, K, topk, window, scale, softcap)


def shape_of(wl) -> focus_shape:
    """focus_shape of an inputs.Workload"""
    return make_shape(wl.Hq, wl.Hkv, wl.n, wl.D, wl.K, wl.topk, wl.window, wl.scale, wl.softcap)


def tensor_arg(t: torch.Tensor) -> focus_tensor:
    """[H, n, D] or [batch, H, n, D] bf16 CUDA tensor with D contiguous"""
    st = t.stride()
    assert t.is_cuda and t.dtype is torch.bfloat16 and st[-1] == 1
    if len(st) == 3:
        return focus_tensor(t.data_ptr(), st[0] * t.shape[0], st[0], st[1])
    assert len(st) == 4
    return focus_tensor(t.data_ptr(), st[0], st[1], st[2])


def focus_version() -> int:
    return lib().focus_version()


def focus_assign(shape, x, H, centroids, masks_out, near_ties=None, near_tie_eps=1e-5, stream=None):
    rc = _short().assign(shape, x, H, centroids, masks_out, near_ties, near_tie_eps, stream)
    if rc is None:
        rc = lib().focus_assign(C.byref(shape), tensor_arg(x), H, _p(centroids), _p(masks_out), _p(near_ties), near_tie_eps, _stream(stream))
    _check(rc)


def focus_assign_hidden(shape, h, Wg, Cg, bias, folded, mq_out, mk_out, near_ties=None, near_tie_eps=1e-5, stream=None):
    """h bf16 [batch, n, d_model] (or [n, d_model]); Wg fp32 [d_model, d_g]; Cg fp32 [K, d_g]; folded fp32 [K, d_model] scratch"""
    rc = _short().assign_hidden(shape, h, Wg, Cg, bias, folded, mq_out, mk_out, near_ties, near_tie_eps, stream)
    if rc is None:
        assert h.is_cuda and h.dtype == torch.bfloat16 and h.stride(-1) == 1
        sb, sn = (h.stride(0), h.stride(1)) if h.dim() == 3 else (h.stride(0) * h.shape[0], h.stride(0))
        rc = lib().focus_assign_hidden(C.byref(shape), _p(h), sb, sn, h.shape[-1], Wg.shape[1], _p(Wg), _p(Cg), _p(bias),
                                       _p(folded), _p(mq_out), _p(mk_out), _p(near_ties), near_tie_eps, _stream(stream))
    _check(rc)


def focus_tiles_layout_of(shape, layout) -> focus_tiles_layout:
    out = focus_tiles_layout()
    _check(lib().focus_tiles_layout_of(C.byref(shape), layout, C.byref(out)))
    return out


def focus_tiles_workspace_bytes(shape, layout) -> int:
    return int(lib().focus_tiles_workspace_bytes(C.byref(shape), layout))


def focus_build_tiles(shape, mq, mk, layout, ws, stream=None):
    rc = _short().build_tiles(shape, mq, mk, layout, ws, stream)
    if rc is None:
        rc = lib().focus_build_tiles(C.byref(shape), _p(mq), _p(mk), layout, _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(rc)


def focus_attn_fwd(shape, q, k, v, mq, mk, tiles_ws, layout, o, lse, dev_status=None, stream=None):
    rc = _short().attn_fwd(shape, q, k, v, mq, mk, tiles_ws, layout, o, lse, dev_status, stream)
    if rc is None:
        rc = lib().focus_attn_fwd(C.byref(shape), tensor_arg(q), tensor_arg(k), tensor_arg(v), _p(mq), _p(mk),
                                  _p(tiles_ws), layout, tensor_arg(o), _p(lse), _p(dev_status), _stream(stream))
    _check(rc)


def focus_decode_workspace_bytes(shape) -> int:
    return int(lib().focus_decode_workspace_bytes(C.byref(shape)))


def focus_decode_step(shape, q, k, v, mq_new, mk, o, lse, ws, stream=None):
    """q, o bf16 [Hq, D] (or [batch, Hq, D]); k, v bf16 caches [Hkv, n, D]; mq_new int32 [batch*Hq]; mk int32 [batch*Hkv, n]"""
    def vec_arg(t):
        st = t.stride()
        assert t.is_cuda and t.dtype is torch.bfloat16 and st[-1] == 1
        if len(st) == 2:
            return focus_tensor(t.data_ptr(), st[0] * t.shape[0], st[0], t.shape[-1])
        return focus_tensor(t.data_ptr(), st[0], st[1], t.shape[-1])
    rc = _short().decode_step(shape, q, k, v, mq_new, mk, o, lse, ws, stream)
    if rc is None:
        rc = lib().focus_decode_step(C.byref(shape), vec_arg(q), tensor_arg(k), tensor_arg(v), _p(mq_new), _p(mk), vec_arg(o),
                                     _p(lse), _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(rc)


def _dev(t, dtype, *shape):
    """the tensor, checked: on the GPU, of this type, contiguous, of this many elements"""
    assert t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.numel() == math.prod(shape), (t.dtype, tuple(t.shape), t.stride(), shape)
    return t.data_ptr()


def _scratch(ws):
    """address and bytes of a workspace, checked: on the GPU, in one piece"""
    assert ws.is_cuda and ws.is_contiguous(), (ws.dtype, tuple(ws.shape), ws.stride())
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _opt(t, dtype, *shape):
    return None if t is None else _dev(t, dtype, *shape)


def _heads(t, shape, H, n=None):
    """tensor_arg of a [batch, H, n, D] tensor (or [H, n, D] for one sequence), with its sizes checked"""
    n = shape.n if n is None else n
    assert tuple(t.shape) == (shape.batch, H, n, shape.D) or (shape.batch == 1 and tuple(t.shape) == (H, n, shape.D)), (tuple(t.shape), (shape.batch, H, n, shape.D))
    st = t.stride()
    assert t.is_cuda and t.dtype is torch.bfloat16 and st[-1] == 1
    # (the stride of a dimension of one element is any number: not used)
    sb, sh, sn = (st[0] if len(st) == 4 and shape.batch > 1 else 0), (st[-3] if H > 1 else shape.D), (st[-2] if n > 1 else shape.D)
    return focus_tensor(t.data_ptr(), sb, sh, sn)


def _vecs(t, shape, H):
    """the argument for [batch, H, D] query or output vectors (or [H, D] for one sequence)"""
    assert tuple(t.shape) == (shape.batch, H, shape.D) or (shape.batch == 1 and tuple(t.shape) == (H, shape.D)), (tuple(t.shape), (shape.batch, H, shape.D))
    st = t.stride()
    assert t.is_cuda and t.dtype is torch.bfloat16 and st[-1] == 1
    return focus_tensor(t.data_ptr(), st[0] if len(st) == 3 and shape.batch > 1 else 0, st[-2] if H > 1 else shape.D, shape.D)


def make_rope(rotary, interleaved=False, amplitude=1.0, eps=1e-6) -> focus_rope:
    return focus_rope(rotary, int(interleaved), amplitude, eps)


def focus_rope_frequencies(rotary, base=10000.0, scaling=FOCUS_ROPE_PLAIN, factor=1.0, low=1.0, high=32.0, trained=1.0, device="cuda"):
    """(float64 tensor [rotary/2] on `device`, amplitude)"""
    out, amplitude = (C.c_double * (max(0, rotary) // 2 + 1))(), C.c_float()
    _check(lib().focus_rope_frequencies(rotary, base, scaling, factor, low, high, trained, C.cast(out, C.c_void_p), C.byref(amplitude)))
    return torch.tensor(out[:rotary // 2], dtype=torch.float64, device=device), amplitude.value


def focus_qk_norm_rope(shape, rope, q, k, wq, wk, freq, positions, q_out, k_out, stream=None):
    """q, q_out bf16 [batch, Hq, n, D], k, k_out [batch, Hkv, n, D] (any strides with D contiguous; the outputs may be the inputs);
    wq, wk fp32 [D] or None; freq fp64 [rotary/2]; positions int32 [batch, n] or None"""
    rc = _short().qk_norm_rope(shape, rope, q, k, wq, wk, freq, positions, q_out, k_out, stream)
    if rc is None:
        D, B, n = shape.D, shape.batch, shape.n
        rc = lib().focus_qk_norm_rope(C.byref(shape), C.byref(rope), _heads(q, shape, shape.Hq), _heads(k, shape, shape.Hkv), _opt(wq, torch.float32, D),
                                      _opt(wk, torch.float32, D), _opt(freq, torch.float64, rope.rotary // 2), _opt(positions, torch.int32, B, n),
                                      _heads(q_out, shape, shape.Hq), _heads(k_out, shape, shape.Hkv), _stream(stream))
    _check(rc)


def focus_qk_norm_rope_bwd_workspace_bytes(shape) -> int:
    return int(lib().focus_qk_norm_rope_bwd_workspace_bytes(C.byref(shape)))


def focus_qk_norm_rope_bwd(shape, rope, q, k, wq, wk, freq, positions, dq_out, dk_out, dq, dk, dwq, dwk, ws, stream=None):
    """gradients dq, dk (bf16, like q and k; may be dq_out, dk_out) and dwq, dwk (fp32 [D]; None where the weight is) from those of the
    results; ws uint8 scratch"""
    rc = _short().qk_norm_rope_bwd(shape, rope, q, k, wq, wk, freq, positions, dq_out, dk_out, dq, dk, dwq, dwk, ws, stream)
    if rc is None:
        D, B, n = shape.D, shape.batch, shape.n
        rc = lib().focus_qk_norm_rope_bwd(C.byref(shape), C.byref(rope), _heads(q, shape, shape.Hq), _heads(k, shape, shape.Hkv),
                                          _opt(wq, torch.float32, D), _opt(wk, torch.float32, D), _opt(freq, torch.float64, rope.rotary // 2),
                                          _opt(positions, torch.int32, B, n), _heads(dq_out, shape, shape.Hq), _heads(dk_out, shape, shape.Hkv),
                                          _heads(dq, shape, shape.Hq), _heads(dk, shape, shape.Hkv), _opt(dwq, torch.float32, D),
                                          _opt(dwk, torch.float32, D), *_scratch(ws), _stream(stream))
    _check(rc)


def focus_kv4_page_bytes(shape, page_tokens) -> int:
    return int(lib().focus_kv4_page_bytes(C.byref(shape), page_tokens))


def make_kv4(pages, page_tokens, table=None, lens=None, k_scale=1.0, v_scale=1.0) -> focus_kv4:
    """pages uint8 [num_pages, focus_kv4_page_bytes]; table int32 [batch, max_pages]; lens int32 [batch].  The struct holds the tensors."""
    assert pages.is_cuda and pages.dtype is torch.uint8 and pages.dim() == 2 and pages.is_contiguous()
    assert (table is None) == (lens is None)
    if table is not None:
        assert table.is_cuda and table.dtype is torch.int32 and table.dim() == 2 and table.is_contiguous()
        assert lens.is_cuda and lens.dtype is torch.int32 and lens.dim() == 1 and lens.is_contiguous() and lens.shape[0] == table.shape[0]
    c = focus_kv4(pages.data_ptr(), _p(table), _p(lens), pages.shape[0], page_tokens, table.shape[1] if table is not None else 0, k_scale, v_scale)
    c.tensors = (pages, table, lens)
    return c


def _fits(cache, shape, paged=True):
    """the cache's tensors against the shape of a call"""
    pages, table, lens = cache.tensors
    want, D = cache.page_tokens, shape.D
    want *= shape.Hkv * (D + D // 8 + 4)
    assert want == pages.shape[1], f"pages of {pages.shape[1]} bytes, {want} for this shape"
    assert not paged or (lens is not None and lens.shape[0] == shape.batch), "table and lens of another batch"


def focus_kv4_append(shape, cache, k, v, mk, counts=None, dev_status=None, stream=None):
    """k, v bf16 [batch, Hkv, n, D] (or [Hkv, n, D]); mk int32 [batch*Hkv, n]; counts int32 [batch] or None"""
    _fits(cache, shape)
    rc = _short().kv4_append(shape, cache, k, v, mk, counts, dev_status, stream)
    if rc is None:
        rc = lib().focus_kv4_append(C.byref(shape), C.byref(cache), _heads(k, shape, shape.Hkv), _heads(v, shape, shape.Hkv),
                                    _dev(mk, torch.int32, shape.batch, shape.Hkv, shape.n), _opt(counts, torch.int32, shape.batch),
                                    _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def focus_kv4_read(shape, cache, first, k, v, mk=None, dev_status=None, stream=None):
    """tokens first[b] .. first[b] + n - 1 (first int32 [batch] or None: from the start) into k, v bf16 [batch, Hkv, n, D] and mk int32 [batch*Hkv, n]"""
    _fits(cache, shape)
    rc = _short().kv4_read(shape, cache, first, k, v, mk, dev_status, stream)
    if rc is None:
        rc = lib().focus_kv4_read(C.byref(shape), C.byref(cache), _opt(first, torch.int32, shape.batch), _heads(k, shape, shape.Hkv),
                                  _heads(v, shape, shape.Hkv), _opt(mk, torch.int32, shape.batch, shape.Hkv, shape.n),
                                  _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def focus_kv4_copy_pages(shape, cache, src, dst, dev_status=None, stream=None):
    """pages src[i] -> dst[i]; int32 lists on the GPU"""
    _fits(cache, shape, False)
    rc = _short().kv4_copy_pages(shape, cache, src, dst, dev_status, stream)
    if rc is None:
        count = src.numel()
        rc = lib().focus_kv4_copy_pages(C.byref(shape), C.byref(cache), _dev(src, torch.int32, count), _dev(dst, torch.int32, count), count,
                                        _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def focus_kv4_decode_workspace_bytes(shape) -> int:
    return int(lib().focus_kv4_decode_workspace_bytes(C.byref(shape)))


def focus_kv4_decode_step(shape, cache, q, mq_new, o, lse, ws, dev_status=None, stream=None):
    """q, o bf16 [batch, Hq, D] (or [Hq, D]); mq_new int32 [batch*Hq]; lse fp32 [batch*Hq]; shape.n bounds the lengths"""
    _fits(cache, shape)
    rc = _short().kv4_decode_step(shape, cache, q, mq_new, o, lse, ws, dev_status, stream)
    if rc is None:
        rc = lib().focus_kv4_decode_step(C.byref(shape), C.byref(cache), _vecs(q, shape, shape.Hq), _dev(mq_new, torch.int32, shape.batch, shape.Hq),
                                         _vecs(o, shape, shape.Hq), _dev(lse, torch.float32, shape.batch, shape.Hq),
                                         *_scratch(ws), _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def focus_soft_ld(K) -> int:
    return int(lib().focus_soft_ld(K))


def focus_router_scores(shape, h, Wg, Cg, folded, scores_out, stream=None):
    """h bf16 [batch, n, d_model] (or [n, d_model]); scores_out fp32 [batch, n, focus_soft_ld(K)]"""
    assert h.is_cuda and h.dtype == torch.bfloat16 and h.stride(-1) == 1
    sb, sn = (h.stride(0), h.stride(1)) if h.dim() == 3 else (h.stride(0) * h.shape[0], h.stride(0))
    _check(lib().focus_router_scores(C.byref(shape), _p(h), sb, sn, h.shape[-1], Wg.shape[1], _p(Wg), _p(Cg), _p(folded),
                                     _p(scores_out), _stream(stream)))


def focus_sinkhorn_workspace_bytes(shape, iters) -> int:
    return int(lib().focus_sinkhorn_workspace_bytes(C.byref(shape), iters))


def focus_sinkhorn(shape, scores, tau, iters, ws, g_out, stream=None):
    """scores, g_out fp32 [batch, n, focus_soft_ld(K)] (may be the same tensor); ws uint8 scratch"""
    _check(lib().focus_sinkhorn(C.byref(shape), _p(scores), tau, iters, _p(ws), ws.numel() * ws.element_size(), _p(g_out),
                                _stream(stream)))


def focus_sinkhorn_bwd_workspace_bytes(shape, iters) -> int:
    return int(lib().focus_sinkhorn_bwd_workspace_bytes(C.byref(shape), iters))


def focus_sinkhorn_bwd(shape, scores, tau, iters, ws, dg, dscores_out, stream=None):
    """scores, dg, dscores_out fp32 [batch, n, focus_soft_ld(K)] (dscores_out may be dg); ws uint8 scratch"""
    _check(lib().focus_sinkhorn_bwd(C.byref(shape), _p(scores), tau, iters, _p(ws), ws.numel() * ws.element_size(), _p(dg),
                                    _p(dscores_out), _stream(stream)))


def focus_gate_attn_fwd(shape, q, k, v, g, lam, o, lse, dev_status=None, stream=None):
    """training-time gated forward; g fp32 [batch, n, focus_soft_ld(K)]"""
    _check(lib().focus_gate_attn_fwd(C.byref(shape), tensor_arg(q), tensor_arg(k), tensor_arg(v), _p(g), lam, tensor_arg(o),
                                     _p(lse), _p(dev_status), _stream(stream)))


def focus_attn_bwd_workspace_bytes(shape) -> int:
    return int(lib().focus_attn_bwd_workspace_bytes(C.byref(shape)))


def focus_attn_bwd(shape, q, k, v, mq, mk, tiles_ws, layout, o, lse, d_o, dq, dk, dv, ws, dev_status=None, stream=None):
    """dq (like q), dk, dv (like k) bf16 from d_o (like o) and what the forward pass left: o, lse fp32 [batch, Hq, n]; ws uint8 scratch"""
    rc = _short().attn_bwd(shape, q, k, v, mq, mk, tiles_ws, layout, o, lse, d_o, dq, dk, dv, ws, dev_status, stream)
    if rc is None:
        B, Hq, Hkv, n = shape.batch, shape.Hq, shape.Hkv, shape.n
        rc = lib().focus_attn_bwd(C.byref(shape), _heads(q, shape, Hq), _heads(k, shape, Hkv), _heads(v, shape, Hkv), _opt(mq, torch.int32, B, Hq, n),
                                  _opt(mk, torch.int32, B, Hkv, n), _p(tiles_ws), layout, _heads(o, shape, Hq), _dev(lse, torch.float32, B, Hq, n),
                                  _heads(d_o, shape, Hq), _heads(dq, shape, Hq), _heads(dk, shape, Hkv), _heads(dv, shape, Hkv), *_scratch(ws),
                                  _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def focus_gate_attn_bwd_workspace_bytes(shape) -> int:
    return int(lib().focus_gate_attn_bwd_workspace_bytes(C.byref(shape)))


def focus_gate_attn_bwd(shape, q, k, v, g, lam, o, lse, d_o, dq, dk, dv, dg, ws, dev_status=None, stream=None):
    """the same for the training-time gate; g, dg fp32 [batch, n, focus_soft_ld(K)]"""
    rc = _short().gate_attn_bwd(shape, q, k, v, g, lam, o, lse, d_o, dq, dk, dv, dg, ws, dev_status, stream)
    if rc is None:
        B, Hq, Hkv, n, ld = shape.batch, shape.Hq, shape.Hkv, shape.n, focus_soft_ld(shape.K)
        rc = lib().focus_gate_attn_bwd(C.byref(shape), _heads(q, shape, Hq), _heads(k, shape, Hkv), _heads(v, shape, Hkv), _dev(g, torch.float32, B, n, ld), lam,
                                       _heads(o, shape, Hq), _dev(lse, torch.float32, B, Hq, n), _heads(d_o, shape, Hq), _heads(dq, shape, Hq),
                                       _heads(dk, shape, Hkv), _heads(dv, shape, Hkv), _dev(dg, torch.float32, B, n, ld), *_scratch(ws),
                                       _opt(dev_status, torch.int32, 4), _stream(stream))
    _check(rc)


def _hidden(t, shape):
    """address and strides of hidden states bf16 [batch, n, d_model] (or [n, d_model] for one sequence)"""
    assert t.is_cuda and t.dtype is torch.bfloat16 and t.stride(-1) == 1, (t.dtype, t.stride())
    d = t.shape[-1]
    assert tuple(t.shape) == (shape.batch, shape.n, d) or (shape.batch == 1 and tuple(t.shape) == (shape.n, d)), (tuple(t.shape), (shape.batch, shape.n, d))
    return t.data_ptr(), t.stride(0) if shape.batch > 1 else 0, t.stride(-2) if shape.n > 1 else d


def focus_router_scores_bwd_workspace_bytes(shape, d_model, d_g) -> int:
    return int(lib().focus_router_scores_bwd_workspace_bytes(C.byref(shape), d_model, d_g))


def focus_router_scores_bwd(shape, h, Wg, Cg, dscores, dh, dWg, dC, ws, stream=None):
    """dh (like h; None: not wanted), dWg fp32 [d_model, d_g], dC fp32 [K, d_g] from dscores fp32 [batch, n, focus_soft_ld(K)]; ws uint8 scratch"""
    rc = _short().router_scores_bwd(shape, h, Wg, Cg, dscores, dh, dWg, dC, ws, stream)
    if rc is None:
        d, dg, K = h.shape[-1], Wg.shape[-1], shape.K
        assert dh is None or dh.shape == h.shape, (tuple(dh.shape), tuple(h.shape))
        ph, pd = _hidden(h, shape), _hidden(dh, shape) if dh is not None else (None, 0, d)
        rc = lib().focus_router_scores_bwd(C.byref(shape), *ph, d, dg, _dev(Wg, torch.float32, d, dg), _dev(Cg, torch.float32, K, dg),
                                           _dev(dscores, torch.float32, shape.batch, shape.n, focus_soft_ld(K)), *pd, _dev(dWg, torch.float32, d, dg),
                                           _dev(dC, torch.float32, K, dg), *_scratch(ws), _stream(stream))
    _check(rc)


def focus_grad_clip_workspace_bytes() -> int:
    return int(lib().focus_grad_clip_workspace_bytes())


def make_grad_list(grads, out=None):
    """the argument of focus_grad_clip: fp32 and bf16 tensors, each contiguous, and where their scaled forms go (None: in place).  The list
    holds the tensors."""
    grads = list(grads)
    out = grads if out is None else list(out)
    assert len(out) == len(grads)
    kinds = {torch.float32: 0, torch.bfloat16: 1}
    entries = (focus_grad * max(1, len(grads)))()
    spans = []
    for e, s, d in zip(entries, grads, out):
        assert s.is_cuda and s.dtype in kinds and s.is_contiguous(), (s.dtype, tuple(s.shape), s.stride())
        assert d.dtype is s.dtype and d.device == s.device == out[0].device and d.is_contiguous() and d.numel() == s.numel(), (d.dtype, tuple(d.shape), d.stride(), "or several devices")
        src, dst, count = s.data_ptr(), d.data_ptr(), s.numel()
        e.src, e.dst, e.count, e.dtype = src, dst, count, kinds[s.dtype]
        if count:
            spans.append((dst, count * s.element_size(), True))
            if src != dst:
                spans.append((src, count * s.element_size(), False))
    # what is written overlaps nothing else: by address, against the furthest ends of what is read and of what is written before it
    read = wrote = last = 0
    for at, size, writes in sorted(spans):
        assert not writes or at != last, "a tensor is listed twice"
        assert at >= wrote and (not writes or at >= read), "a tensor is written over another"
        if writes:
            wrote, last = max(wrote, at + size), at
        else:
            read = max(read, at + size)
    c = focus_grads(C.addressof(entries), len(grads))
    c.tensors = (entries, grads, out)
    return c


def focus_grad_clip(grads, max_norm, norm_out, ws, stream=None):
    """grads from make_grad_list; norm_out fp32 [1] or None; ws uint8 scratch"""
    rc = _short().grad_clip(grads, max_norm, norm_out, ws, stream)
    if rc is None:
        rc = lib().focus_grad_clip(grads.grads, grads.count, max_norm, _opt(norm_out, torch.float32, 1), *_scratch(ws), _stream(stream))
    _check(rc)


def focus_count_kept(shape, mq, tiles_ws, counts_out, stream=None):
    _check(lib().focus_count_kept(C.byref(shape), _p(mq), _p(tiles_ws), _p(counts_out), _stream(stream)))


def focus_count_kept_noalloc(shape, mq, mk, counts_out, stream=None):
    """focus_count_kept for callers that may not allocate: the group bitmaps go to an array built into the
    library (at most 1 MiB: batch*Hkv*ceil(n/128)*K*16 bytes), no workspace argument."""
    _check(lib().focus_count_kept_noalloc(C.byref(shape), _p(mq), _p(mk), _p(counts_out), _stream(stream)))


def focus_selftest_umma(D, a, b, p, v, s_out, o_out, dev_status, stream=None):
    _check(lib().focus_selftest_umma(D, _p(a), _p(b), _p(p), _p(v), _p(s_out), _p(o_out), _p(dev_status),
                                     _stream(stream)))


def focus_selftest_umma_pair(a, b, p, v, s_out, o_out, dev_status, stream=None):
    _check(lib().focus_selftest_umma_pair(_p(a), _p(b), _p(p), _p(v), _p(s_out), _p(o_out), _p(dev_status), _stream(stream)))


def focus_selftest_mma_rate(pair, N, ts, pattern, rounds, result, stream=None):
    """result: int64 device tensor of 3 words (cycles, nanoseconds, fault flag)"""
    _check(lib().focus_selftest_mma_rate(pair, N, ts, pattern, rounds, _p(result), _stream(stream)))


def focus_selftest_stalled_wait(shape, q, k, v, o, lse, wait_limit_ns, dev_status, stream=None):
    _check(lib().focus_selftest_stalled_wait(C.byref(shape), tensor_arg(q), tensor_arg(k), tensor_arg(v), tensor_arg(o), _p(lse),
                                             wait_limit_ns, _p(dev_status), _stream(stream)))


def focus_selftest_stalled_exchange(shape, scores, tau, iters, ws, wait_limit_cycles, stall_at, g_out, stream=None):
    _check(lib().focus_selftest_stalled_exchange(C.byref(shape), _p(scores), tau, iters, _p(ws), ws.numel() * ws.element_size(),
                                                 wait_limit_cycles, stall_at, _p(g_out), _stream(stream)))


def alloc_workspace(shape, layout, device="cuda") -> torch.Tensor:
    """uint8 device buffer of focus_tiles_workspace_bytes (torch allocations are 256-byte aligned)"""
    nbytes = focus_tiles_workspace_bytes(shape, layout)
    if nbytes == 0:
        raise FocusError(-1, lib().focus_last_error().decode())
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def ws_view(ws: torch.Tensor, offset: int, count: int, dtype) -> torch.Tensor:
    """typed view of `count` elements at byte `offset` of a workspace"""
    size = torch.empty((), dtype=dtype).element_size()
    return ws[offset:offset + count * size].view(dtype)
