// The short calls of binding.py without ctypes: tensors to addresses and strides, the current stream, the call.
//
// A decode step or a prompt of a thousand tokens takes the GPU 15 to 30 us, and marshalling the arguments of its three or four
// calls through ctypes took the host as long: 8 us a focus_assign and 16 a focus_decode_step on a slow core.  A decode step over
// 2049 keys in a row of them: 33.0 -> 21.4 us (30.6 -> 19.4 on a faster host); from the call until the GPU is done, with the GPU
// idle before: 45.5 -> 34.3, and a prompt of 1024 tokens in buffers not used before 65 -> 48.  The calls around the 4-bit cache, which
// check their tensors' sizes too, among others of their kind: a token of 16 sequences through focus_qk_norm_rope 11.7 -> 3.2 us, a token of 32
// sequences stored and read back 19 -> 6.6, 48 pages copied 8.5 -> 4.8.
//
// The functions take what binding.py's take.  They answer None when an argument is none that they know how to read (a tensor
// subclass, a shape that is no focus_shape, ...), before anything has been enqueued; binding.py then goes through ctypes as for
// its other entry points.
#include <Python.h>

#include <optional>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "focus.h"

namespace {

PyObject* shape_type;                // binding.focus_shape
PyObject *rope_type, *kv4_type;      // binding.focus_rope, binding.focus_kv4
PyObject* grads_type;                // binding.focus_grads
struct Grads {                       // its layout
    const focus_grad* grads;
    int32_t count;
};

// The entry points, from the library that binding.py has loaded: linked against, the loader might find another copy of it.
decltype(&focus_assign) p_assign;
decltype(&focus_assign_hidden) p_assign_hidden;
decltype(&focus_build_tiles) p_build_tiles;
decltype(&focus_attn_fwd) p_attn_fwd;
decltype(&focus_decode_step) p_decode_step;
decltype(&focus_qk_norm_rope) p_qk_norm_rope;
decltype(&focus_qk_norm_rope_bwd) p_qk_norm_rope_bwd;
decltype(&focus_kv4_append) p_kv4_append;
decltype(&focus_kv4_read) p_kv4_read;
decltype(&focus_kv4_copy_pages) p_kv4_copy_pages;
decltype(&focus_kv4_decode_step) p_kv4_decode_step;
decltype(&focus_attn_bwd) p_attn_bwd;
decltype(&focus_gate_attn_bwd) p_gate_attn_bwd;
decltype(&focus_router_scores_bwd) p_router_scores_bwd;
decltype(&focus_grad_clip) p_grad_clip;

struct Args {
    PyObject* const* a;
    bool known = true;               // every argument so far was of a kind that is read here
    bool failed = false;             // a Python error is set

    template <class T>
    const T* object(int i, PyObject* type) {
        Py_buffer b;
        if (!known || failed || (PyObject*)Py_TYPE(a[i]) != type) { known = false; return nullptr; }
        if (PyObject_GetBuffer(a[i], &b, PyBUF_SIMPLE)) { failed = true; return nullptr; }
        const T* s = b.len == (Py_ssize_t)sizeof(T) ? static_cast<const T*>(b.buf) : nullptr;
        PyBuffer_Release(&b);        // (the caller's reference keeps the object, and with it the memory)
        if (!s) known = false;
        return s;
    }
    const focus_shape* shape(int i) { return object<focus_shape>(i, shape_type); }
    const at::Tensor* tensor(int i) {
        if (!known || failed || !THPVariable_CheckExact(a[i])) { known = false; return nullptr; }
        return &THPVariable_Unpack(a[i]);
    }
    // address of a tensor, or of nothing
    void* ptr(int i) {
        if (!known || failed || a[i] == Py_None) return nullptr;
        const at::Tensor* t = tensor(i);
        return t ? t->data_ptr() : nullptr;
    }
    // [H, n, D] or [batch, H, n, D] bf16 CUDA tensor with D contiguous; `vector`: [H, D] or [batch, H, D]
    focus_tensor bf16(int i, bool vector) {
        focus_tensor out = {};
        const at::Tensor* t = tensor(i);
        if (!t) return out;
        const int dims = (int)t->dim(), outer = vector ? 1 : 2;
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || (dims != outer + 1 && dims != outer + 2) || t->stride(dims - 1) != 1) {
            known = false;           // binding.py says what is wrong with it
            return out;
        }
        const int h = dims - outer - 1;                  // dimension of the heads
        out.ptr = t->data_ptr();
        out.stride_h = t->stride(h);
        out.stride_b = h == 0 ? out.stride_h * t->size(0) : t->stride(0);
        out.stride_n = vector ? t->size(dims - 1) : t->stride(h + 1);
        return out;
    }
    // the same with its sizes checked against the shape: [batch, H, n, D], or without `batch` for one sequence (`vector`: without n)
    focus_tensor sized(int i, const focus_shape* s, int H, bool vector) {
        focus_tensor out = {};
        const at::Tensor* t = tensor(i);
        if (!t || !s) { known = false; return out; }
        const int dims = (int)t->dim(), own = vector ? 2 : 3, h = dims - own;
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || (h != 1 && !(h == 0 && s->batch == 1)) || (h == 1 && t->size(0) != s->batch) ||
            t->size(h) != H || (!vector && t->size(h + 1) != s->n) || t->size(dims - 1) != s->D || t->stride(dims - 1) != 1) {
            known = false;           // binding.py says what is wrong with it
            return out;
        }
        out.ptr = t->data_ptr();     // (the stride of a dimension of one element is any number: not used)
        out.stride_b = h == 1 && s->batch > 1 ? t->stride(0) : 0;
        out.stride_h = H > 1 ? t->stride(h) : s->D;
        out.stride_n = !vector && s->n > 1 ? t->stride(h + 1) : s->D;
        return out;
    }
    // address of a contiguous tensor of this many elements on the GPU; None where `optional`
    void* counted(int i, at::ScalarType type, int64_t count, bool optional) {
        if (!known || failed || (optional && a[i] == Py_None)) return nullptr;
        const at::Tensor* t = tensor(i);
        if (!t || !t->is_cuda() || t->scalar_type() != type || t->numel() != count || !t->is_contiguous()) { known = false; return nullptr; }
        return t->data_ptr();
    }
    // hidden states bf16 [batch, n, d] (or [n, d] for one sequence); their `d`
    focus_tensor hidden(int i, const focus_shape* s, int64_t& d) {
        focus_tensor out = {};
        const at::Tensor* t = tensor(i);
        if (!t || !s) { known = false; return out; }
        const int dims = (int)t->dim();
        if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || (dims != 3 && !(dims == 2 && s->batch == 1)) || t->stride(dims - 1) != 1 ||
            (dims == 3 && t->size(0) != s->batch) || t->size(dims - 2) != s->n || t->size(dims - 1) > INT32_MAX) {
            known = false;
            return out;
        }
        d = t->size(dims - 1);
        out.ptr = t->data_ptr();
        out.stride_b = s->batch > 1 ? t->stride(0) : 0;
        out.stride_n = s->n > 1 ? t->stride(dims - 2) : d;
        return out;
    }
    // address of a workspace on the GPU, in one piece
    void* scratch(int i) {
        const at::Tensor* t = tensor(i);
        if (!t || !t->is_cuda() || !t->is_contiguous()) { known = false; return nullptr; }
        return t->data_ptr();
    }
    size_t bytes(int i) {
        const at::Tensor* t = tensor(i);
        return t ? (size_t)t->numel() * t->element_size() : 0;
    }
    int32_t integer(int i) {
        if (!known || failed) return 0;
        if (!PyLong_CheckExact(a[i])) { known = false; return 0; }
        int over = 0;
        const long v = PyLong_AsLongAndOverflow(a[i], &over);
        if (over || v != (int32_t)v) known = false;
        return (int32_t)v;
    }
    float number(int i) {
        if (!known || failed) return 0.f;
        if (!PyFloat_CheckExact(a[i])) { known = false; return 0.f; }
        return (float)PyFloat_AS_DOUBLE(a[i]);
    }
    void* stream(int i) {
        if (!known || failed) return nullptr;
        if (a[i] != Py_None) { known = false; return nullptr; }
        return c10::cuda::getCurrentCUDAStream().stream();
    }
};

// `read` reads the arguments and returns the call to make
template <class Read>
PyObject* enter(PyObject* const* args, Py_ssize_t got, Py_ssize_t want, Read read) {
    if (got != want) return PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", got, want);
    Args a{args};
    auto guarded = [&]() -> decltype(std::make_optional(read(a))) {
        try {
            return read(a);
        } catch (const std::exception&) {                // a tensor without storage, no driver, ...: binding.py meets it again
            a.known = false;
            return std::nullopt;
        }
    };
    auto call = guarded();
    if (a.failed) return nullptr;
    if (!a.known || !call) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = (*call)();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject* assign(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 8, [](Args& a) {
        auto s = a.shape(0);
        auto x = a.bf16(1, false);
        auto H = a.integer(2);
        auto c = static_cast<const float*>(a.ptr(3));
        auto m = static_cast<uint32_t*>(a.ptr(4));
        auto near = static_cast<unsigned long long*>(a.ptr(5));
        auto eps = a.number(6);
        auto st = a.stream(7);
        return [=] { return p_assign(s, x, H, c, m, near, eps, st); };
    });
}

PyObject* assign_hidden(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 11, [](Args& a) {
        auto s = a.shape(0);
        focus_tensor h = {};                             // [n, d_model] or [batch, n, d_model]
        int32_t d = 0, dg = 0;
        if (const at::Tensor* t = a.tensor(1)) {
            if (t->is_cuda() && t->scalar_type() == at::kBFloat16 && (t->dim() == 2 || t->dim() == 3) && t->stride(-1) == 1) {
                h.ptr = t->data_ptr();
                h.stride_n = t->stride(-2);
                h.stride_b = t->dim() == 3 ? t->stride(0) : t->stride(0) * t->size(0);
                d = (int32_t)t->size(-1);
            } else {
                a.known = false;
            }
        }
        if (const at::Tensor* t = a.tensor(2)) {
            if (t->dim() == 2) dg = (int32_t)t->size(1);
            else a.known = false;
        }
        auto Wg = static_cast<const float*>(a.ptr(2)), Cg = static_cast<const float*>(a.ptr(3)), bias = static_cast<const float*>(a.ptr(4));
        auto folded = static_cast<float*>(a.ptr(5));
        auto mq = static_cast<uint32_t*>(a.ptr(6)), mk = static_cast<uint32_t*>(a.ptr(7));
        auto near = static_cast<unsigned long long*>(a.ptr(8));
        auto eps = a.number(9);
        auto st = a.stream(10);
        return [=] { return p_assign_hidden(s, h.ptr, h.stride_b, h.stride_n, d, dg, Wg, Cg, bias, folded, mq, mk, near, eps, st); };
    });
}

PyObject* build_tiles(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 6, [](Args& a) {
        auto s = a.shape(0);
        auto mq = static_cast<const uint32_t*>(a.ptr(1));
        auto mk = static_cast<const uint32_t*>(a.ptr(2));
        auto layout = a.integer(3);
        auto ws = a.ptr(4);
        auto bytes = a.bytes(4);
        auto st = a.stream(5);
        return [=] { return p_build_tiles(s, mq, mk, layout, ws, bytes, st); };
    });
}

PyObject* attn_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 12, [](Args& a) {
        auto s = a.shape(0);
        auto q = a.bf16(1, false), k = a.bf16(2, false), v = a.bf16(3, false);
        auto mq = static_cast<const uint32_t*>(a.ptr(4));
        auto mk = static_cast<const uint32_t*>(a.ptr(5));
        auto ws = a.ptr(6);
        auto layout = a.integer(7);
        auto o = a.bf16(8, false);
        auto lse = static_cast<float*>(a.ptr(9));
        auto status = static_cast<int32_t*>(a.ptr(10));
        auto st = a.stream(11);
        return [=] { return p_attn_fwd(s, q, k, v, mq, mk, ws, layout, o, lse, status, st); };
    });
}

PyObject* decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 10, [](Args& a) {
        auto s = a.shape(0);
        auto q = a.bf16(1, true);
        auto k = a.bf16(2, false), v = a.bf16(3, false);
        auto mq = static_cast<const uint32_t*>(a.ptr(4));
        auto mk = static_cast<const uint32_t*>(a.ptr(5));
        auto o = a.bf16(6, true);
        auto lse = static_cast<float*>(a.ptr(7));
        auto ws = a.ptr(8);
        auto bytes = a.bytes(8);
        auto st = a.stream(9);
        return [=] { return p_decode_step(s, q, k, v, mq, mk, o, lse, ws, bytes, st); };
    });
}

PyObject* qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 11, [](Args& a) {
        auto s = a.shape(0);
        auto r = a.object<focus_rope>(1, rope_type);
        const int Hq = s ? s->Hq : 0, Hkv = s ? s->Hkv : 0, D = s ? s->D : 0;
        auto q = a.sized(2, s, Hq, false), k = a.sized(3, s, Hkv, false);
        auto wq = static_cast<const float*>(a.counted(4, at::kFloat, D, true)), wk = static_cast<const float*>(a.counted(5, at::kFloat, D, true));
        auto freq = static_cast<const double*>(a.counted(6, at::kDouble, r ? r->rotary / 2 : 0, true));
        auto pos = static_cast<const int32_t*>(a.counted(7, at::kInt, s ? (int64_t)s->batch * s->n : 0, true));
        auto qo = a.sized(8, s, Hq, false), ko = a.sized(9, s, Hkv, false);
        auto st = a.stream(10);
        return [=] { return p_qk_norm_rope(s, r, q, k, wq, wk, freq, pos, qo, ko, st); };
    });
}

PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 16, [](Args& a) {
        auto s = a.shape(0);
        auto r = a.object<focus_rope>(1, rope_type);
        const int Hq = s ? s->Hq : 0, Hkv = s ? s->Hkv : 0, D = s ? s->D : 0;
        auto q = a.sized(2, s, Hq, false), k = a.sized(3, s, Hkv, false);
        auto wq = static_cast<const float*>(a.counted(4, at::kFloat, D, true)), wk = static_cast<const float*>(a.counted(5, at::kFloat, D, true));
        auto freq = static_cast<const double*>(a.counted(6, at::kDouble, r ? r->rotary / 2 : 0, true));
        auto pos = static_cast<const int32_t*>(a.counted(7, at::kInt, s ? (int64_t)s->batch * s->n : 0, true));
        auto gq = a.sized(8, s, Hq, false), gk = a.sized(9, s, Hkv, false), dq = a.sized(10, s, Hq, false), dk = a.sized(11, s, Hkv, false);
        auto dwq = static_cast<float*>(a.counted(12, at::kFloat, D, true)), dwk = static_cast<float*>(a.counted(13, at::kFloat, D, true));
        auto ws = a.scratch(14);
        auto bytes = a.bytes(14);
        auto st = a.stream(15);
        return [=] { return p_qk_norm_rope_bwd(s, r, q, k, wq, wk, freq, pos, gq, gk, dq, dk, dwq, dwk, ws, bytes, st); };
    });
}

PyObject* kv4_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 8, [](Args& a) {
        auto s = a.shape(0);
        auto c = a.object<focus_kv4>(1, kv4_type);
        const int Hkv = s ? s->Hkv : 0, B = s ? s->batch : 0;
        auto k = a.sized(2, s, Hkv, false), v = a.sized(3, s, Hkv, false);
        auto mk = static_cast<const uint32_t*>(a.counted(4, at::kInt, s ? (int64_t)B * Hkv * s->n : 0, false));
        auto counts = static_cast<const int32_t*>(a.counted(5, at::kInt, B, true));
        auto status = static_cast<int32_t*>(a.counted(6, at::kInt, 4, true));
        auto st = a.stream(7);
        return [=] { return p_kv4_append(s, c, k, v, mk, counts, status, st); };
    });
}

PyObject* kv4_read(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 8, [](Args& a) {
        auto s = a.shape(0);
        auto c = a.object<focus_kv4>(1, kv4_type);
        const int Hkv = s ? s->Hkv : 0, B = s ? s->batch : 0;
        auto first = static_cast<const int32_t*>(a.counted(2, at::kInt, B, true));
        auto k = a.sized(3, s, Hkv, false), v = a.sized(4, s, Hkv, false);
        auto mk = static_cast<uint32_t*>(a.counted(5, at::kInt, s ? (int64_t)B * Hkv * s->n : 0, true));
        auto status = static_cast<int32_t*>(a.counted(6, at::kInt, 4, true));
        auto st = a.stream(7);
        return [=] { return p_kv4_read(s, c, first, k, v, mk, status, st); };
    });
}

PyObject* kv4_copy_pages(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 6, [](Args& a) {
        auto s = a.shape(0);
        auto c = a.object<focus_kv4>(1, kv4_type);
        const at::Tensor* t = a.tensor(2);
        const int64_t count = t ? t->numel() : 0;
        if (count > INT32_MAX) a.known = false;
        auto src = static_cast<const int32_t*>(a.counted(2, at::kInt, count, false)), dst = static_cast<const int32_t*>(a.counted(3, at::kInt, count, false));
        auto status = static_cast<int32_t*>(a.counted(4, at::kInt, 4, true));
        auto st = a.stream(5);
        return [=] { return p_kv4_copy_pages(s, c, src, dst, (int32_t)count, status, st); };
    });
}

PyObject* kv4_decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 9, [](Args& a) {
        auto s = a.shape(0);
        auto c = a.object<focus_kv4>(1, kv4_type);
        const int Hq = s ? s->Hq : 0;
        const int64_t vectors = s ? (int64_t)s->batch * Hq : 0;
        auto q = a.sized(2, s, Hq, true);
        auto mq = static_cast<const uint32_t*>(a.counted(3, at::kInt, vectors, false));
        auto o = a.sized(4, s, Hq, true);
        auto lse = static_cast<float*>(a.counted(5, at::kFloat, vectors, false));
        auto ws = a.scratch(6);
        auto bytes = a.bytes(6);
        auto status = static_cast<int32_t*>(a.counted(7, at::kInt, 4, true));
        auto st = a.stream(8);
        return [=] { return p_kv4_decode_step(s, c, q, mq, o, lse, ws, bytes, status, st); };
    });
}

int soft_ld(int K) { return K <= 4 ? 4 : K <= 8 ? 8 : K <= 16 ? 16 : 32; }

PyObject* attn_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 17, [](Args& a) {
        auto s = a.shape(0);
        const int Hq = s ? s->Hq : 0, Hkv = s ? s->Hkv : 0;
        const int64_t rows = s ? (int64_t)s->batch * s->n : 0;
        auto q = a.sized(1, s, Hq, false), k = a.sized(2, s, Hkv, false), v = a.sized(3, s, Hkv, false);
        auto mq = static_cast<const uint32_t*>(a.counted(4, at::kInt, rows * Hq, true)), mk = static_cast<const uint32_t*>(a.counted(5, at::kInt, rows * Hkv, true));
        auto tiles = a.ptr(6);
        auto layout = a.integer(7);
        auto o = a.sized(8, s, Hq, false);
        auto lse = static_cast<const float*>(a.counted(9, at::kFloat, rows * Hq, false));
        auto d_o = a.sized(10, s, Hq, false), dq = a.sized(11, s, Hq, false), dk = a.sized(12, s, Hkv, false), dv = a.sized(13, s, Hkv, false);
        auto ws = a.scratch(14);
        auto bytes = a.bytes(14);
        auto status = static_cast<int32_t*>(a.counted(15, at::kInt, 4, true));
        auto st = a.stream(16);
        return [=] { return p_attn_bwd(s, q, k, v, mq, mk, tiles, layout, o, lse, d_o, dq, dk, dv, ws, bytes, status, st); };
    });
}

PyObject* gate_attn_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 16, [](Args& a) {
        auto s = a.shape(0);
        const int Hq = s ? s->Hq : 0, Hkv = s ? s->Hkv : 0;
        const int64_t rows = s ? (int64_t)s->batch * s->n : 0, ld = s ? soft_ld(s->K) : 0;
        auto q = a.sized(1, s, Hq, false), k = a.sized(2, s, Hkv, false), v = a.sized(3, s, Hkv, false);
        auto g = static_cast<const float*>(a.counted(4, at::kFloat, rows * ld, false));
        auto lam = a.number(5);
        auto o = a.sized(6, s, Hq, false);
        auto lse = static_cast<const float*>(a.counted(7, at::kFloat, rows * Hq, false));
        auto d_o = a.sized(8, s, Hq, false), dq = a.sized(9, s, Hq, false), dk = a.sized(10, s, Hkv, false), dv = a.sized(11, s, Hkv, false);
        auto dg = static_cast<float*>(a.counted(12, at::kFloat, rows * ld, false));
        auto ws = a.scratch(13);
        auto bytes = a.bytes(13);
        auto status = static_cast<int32_t*>(a.counted(14, at::kInt, 4, true));
        auto st = a.stream(15);
        return [=] { return p_gate_attn_bwd(s, q, k, v, g, lam, o, lse, d_o, dq, dk, dv, dg, ws, bytes, status, st); };
    });
}

PyObject* router_scores_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 10, [](Args& a) {
        auto s = a.shape(0);
        int64_t d = 0, dd = 0, dg = 0;
        const int K = s ? s->K : 0;
        auto h = a.hidden(1, s, d);
        if (const at::Tensor* t = a.tensor(2)) {
            if (t->dim() == 2 && t->size(1) <= INT32_MAX) dg = t->size(1);
            else a.known = false;
        }
        auto Wg = static_cast<const float*>(a.counted(2, at::kFloat, d * dg, false)), Cg = static_cast<const float*>(a.counted(3, at::kFloat, K * dg, false));
        auto ds = static_cast<const float*>(a.counted(4, at::kFloat, s ? (int64_t)s->batch * s->n * soft_ld(K) : 0, false));
        focus_tensor dh = {};
        if (a.known && !a.failed && a.a[5] != Py_None) {
            dh = a.hidden(5, s, dd);
            if (dd != d) a.known = false;
        }
        auto dWg = static_cast<float*>(a.counted(6, at::kFloat, d * dg, false)), dC = static_cast<float*>(a.counted(7, at::kFloat, K * dg, false));
        auto ws = a.scratch(8);
        auto bytes = a.bytes(8);
        auto st = a.stream(9);
        return [=] { return p_router_scores_bwd(s, h.ptr, h.stride_b, h.stride_n, (int32_t)d, (int32_t)dg, Wg, Cg, ds, dh.ptr, dh.stride_b, dh.stride_n, dWg, dC, ws, bytes, st); };
    });
}

PyObject* grad_clip(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return enter(args, n, 5, [](Args& a) {
        auto g = a.object<Grads>(0, grads_type);
        auto bound = a.number(1);
        auto norm = static_cast<float*>(a.counted(2, at::kFloat, 1, true));
        auto ws = a.scratch(3);
        auto bytes = a.bytes(3);
        auto st = a.stream(4);
        const Grads list = g ? *g : Grads{};
        return [=] { return p_grad_clip(list.grads, list.count, bound, norm, ws, bytes, st); };
    });
}

// init(type of a shape, addresses of the entry points in the order above)
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 6) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 6", n);
    void* at[5];
    for (int i = 0; i < 5; ++i) {
        at[i] = PyLong_AsVoidPtr(args[1 + i]);
        if (!at[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
    }
    p_assign = reinterpret_cast<decltype(p_assign)>(at[0]);
    p_assign_hidden = reinterpret_cast<decltype(p_assign_hidden)>(at[1]);
    p_build_tiles = reinterpret_cast<decltype(p_build_tiles)>(at[2]);
    p_attn_fwd = reinterpret_cast<decltype(p_attn_fwd)>(at[3]);
    p_decode_step = reinterpret_cast<decltype(p_decode_step)>(at[4]);
    Py_INCREF(args[0]);
    Py_XSETREF(shape_type, args[0]);
    Py_RETURN_NONE;
}

// init_kv4(types of a rotation and of a cache, addresses of the entry points from qk_norm_rope on)
PyObject* init_kv4(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 8) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 8", n);
    void* at[6];
    for (int i = 0; i < 6; ++i) {
        at[i] = PyLong_AsVoidPtr(args[2 + i]);
        if (!at[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
    }
    p_qk_norm_rope = reinterpret_cast<decltype(p_qk_norm_rope)>(at[0]);
    p_qk_norm_rope_bwd = reinterpret_cast<decltype(p_qk_norm_rope_bwd)>(at[1]);
    p_kv4_append = reinterpret_cast<decltype(p_kv4_append)>(at[2]);
    p_kv4_read = reinterpret_cast<decltype(p_kv4_read)>(at[3]);
    p_kv4_copy_pages = reinterpret_cast<decltype(p_kv4_copy_pages)>(at[4]);
    p_kv4_decode_step = reinterpret_cast<decltype(p_kv4_decode_step)>(at[5]);
    Py_INCREF(args[0]);
    Py_XSETREF(rope_type, args[0]);
    Py_INCREF(args[1]);
    Py_XSETREF(kv4_type, args[1]);
    Py_RETURN_NONE;
}

// init_bwd(type of a list of gradients, addresses of the entry points from attn_bwd on)
PyObject* init_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 5", n);
    void* at[4];
    for (int i = 0; i < 4; ++i) {
        at[i] = PyLong_AsVoidPtr(args[1 + i]);
        if (!at[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
    }
    p_attn_bwd = reinterpret_cast<decltype(p_attn_bwd)>(at[0]);
    p_gate_attn_bwd = reinterpret_cast<decltype(p_gate_attn_bwd)>(at[1]);
    p_router_scores_bwd = reinterpret_cast<decltype(p_router_scores_bwd)>(at[2]);
    p_grad_clip = reinterpret_cast<decltype(p_grad_clip)>(at[3]);
    Py_INCREF(args[0]);
    Py_XSETREF(grads_type, args[0]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void*)init, METH_FASTCALL, nullptr},
    {"assign", (PyCFunction)(void*)assign, METH_FASTCALL, nullptr},
    {"assign_hidden", (PyCFunction)(void*)assign_hidden, METH_FASTCALL, nullptr},
    {"build_tiles", (PyCFunction)(void*)build_tiles, METH_FASTCALL, nullptr},
    {"attn_fwd", (PyCFunction)(void*)attn_fwd, METH_FASTCALL, nullptr},
    {"decode_step", (PyCFunction)(void*)decode_step, METH_FASTCALL, nullptr},
    {"init_kv4", (PyCFunction)(void*)init_kv4, METH_FASTCALL, nullptr},
    {"qk_norm_rope", (PyCFunction)(void*)qk_norm_rope, METH_FASTCALL, nullptr},
    {"qk_norm_rope_bwd", (PyCFunction)(void*)qk_norm_rope_bwd, METH_FASTCALL, nullptr},
    {"kv4_append", (PyCFunction)(void*)kv4_append, METH_FASTCALL, nullptr},
    {"kv4_read", (PyCFunction)(void*)kv4_read, METH_FASTCALL, nullptr},
    {"kv4_copy_pages", (PyCFunction)(void*)kv4_copy_pages, METH_FASTCALL, nullptr},
    {"kv4_decode_step", (PyCFunction)(void*)kv4_decode_step, METH_FASTCALL, nullptr},
    {"init_bwd", (PyCFunction)(void*)init_bwd, METH_FASTCALL, nullptr},
    {"attn_bwd", (PyCFunction)(void*)attn_bwd, METH_FASTCALL, nullptr},
    {"gate_attn_bwd", (PyCFunction)(void*)gate_attn_bwd, METH_FASTCALL, nullptr},
    {"router_scores_bwd", (PyCFunction)(void*)router_scores_bwd, METH_FASTCALL, nullptr},
    {"grad_clip", (PyCFunction)(void*)grad_clip, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "short calls of binding.py", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    // the torch and the Python whose objects the code above reads; binding.py compares before it passes it any
    if (m && PyModule_AddStringConstant(m, "built_for", FOCUS_BUILT_FOR)) Py_CLEAR(m);
    return m;
}
