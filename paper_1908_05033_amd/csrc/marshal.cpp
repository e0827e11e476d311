// Argument marshalling of binding.py in native code.
//
// Small layers wait for the host: checking a call's three to seven tensors, asking PyTorch for the
// current stream and passing a dozen arguments through ctypes took 5 of the 7.5 us of a call.  Each
// function here takes the arguments of the binding function of the same name in its order and
// either calls the library and returns the status, or returns None, having done nothing, where an
// argument is not of the plain form that it knows: then the binding takes its general path, which
// converts the argument or refuses it.  Plain are: device tensors of the right dtype, contiguous, of
// type torch.Tensor or Parameter and not wrapped by a transform; int, float and bool objects;
// None or an int address where the general path takes one; a dsq_conv_desc; for the language-model calls, tensors of the
// current device whose shapes, types and strides the general path would accept.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/hip/HIPStream.h>

#include <limits.h>
#include <string.h>

#include <algorithm>

#include "../../include/dsqconv.h"

namespace {

decltype(&dsq_quantize_act) f_quantize_act;
decltype(&dsq_conv2d) f_conv2d;
decltype(&dsq_conv2d_requant) f_conv2d_requant;
decltype(&dsq_conv2d_wq) f_conv2d_wq;
decltype(&dsq_soft_quantize_fwd) f_soft_fwd;
decltype(&dsq_soft_quantize_bwd) f_soft_bwd;
decltype(&dsq_rms_norm) f_rms_norm;
decltype(&dsq_rms_norm_bwd) f_rms_norm_bwd;
decltype(&dsq_linear_w4) f_linear_w4;
decltype(&dsq_linear_w4a8) f_linear_w4a8;
decltype(&dsq_code_row_bytes) f_code_row_bytes;
decltype(&dsq_w4_packed_bytes) f_w4_packed_bytes;
decltype(&dsq_w4_scale_bytes) f_w4_scale_bytes;
decltype(&dsq_qk_norm_rope) f_qk_norm_rope;
decltype(&dsq_qk_norm_rope_bwd) f_qk_norm_rope_bwd;
decltype(&dsq_attention) f_attention;
decltype(&dsq_attention_bwd) f_attention_bwd;
decltype(&dsq_attention_cache) f_attention_cache;
PyTypeObject *desc_type;

// Reads arguments one after the other; `plain` turns false at the first that is not.
struct Args {
    PyObject *const *at;
    bool plain;

    Args(PyObject *const *args, Py_ssize_t given, Py_ssize_t expected)
        : at(args), plain(given == expected && f_quantize_act && !at::impl::torch_function_mode_enabled())
    {
    }
    long long number()
    {
        PyObject *o = *at++;
        if (!plain || !(PyLong_CheckExact(o) || PyBool_Check(o))) { plain = false; return 0; }
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        if (overflow || v < INT_MIN || v > INT_MAX) plain = false;
        return v;
    }
    int integer() { return (int)number(); }
    float real()
    {
        PyObject *o = *at;
        if (plain && PyFloat_CheckExact(o)) { ++at; return (float)PyFloat_AS_DOUBLE(o); }
        return (float)number();
    }
    int truth()
    {
        PyObject *o = *at++;
        if (o != Py_True && o != Py_False) plain = false;
        return o == Py_True;
    }
    void *tensor(at::ScalarType type, bool may_be_none = false, size_t *numel = nullptr)
    {
        PyObject *o = *at++;
        if (!plain) return nullptr;
        if (may_be_none && o == Py_None) return nullptr;
        if (numel == nullptr && PyLong_CheckExact(o)) {                       // a raw device address
            void *p = PyLong_AsVoidPtr(o);
            if (PyErr_Occurred()) { PyErr_Clear(); plain = false; }
            return p;
        }
        plain = false;
        if (!THPVariable_CheckTypeExact(Py_TYPE(o))) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || at::isTensorSubclassLike(t) || !t.has_storage() || !t.is_cuda() || t.scalar_type() != type ||
            !t.is_contiguous())
            return nullptr;
        plain = true;
        if (numel) *numel = (size_t)t.numel();
        return t.data_ptr();
    }
    // A plain device tensor of the current device at the next place, nullptr for None or with `plain` turned false.
    const at::Tensor *here(bool may_be_none)
    {
        PyObject *o = *at++;
        if (!plain || (may_be_none && o == Py_None)) return nullptr;
        plain = false;
        if (!THPVariable_CheckTypeExact(Py_TYPE(o))) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || at::isTensorSubclassLike(t) || !t.has_storage() || !t.is_cuda() || t.get_device() != c10::hip::current_device())
            return nullptr;
        plain = true;
        return &t;
    }
    struct Rows {
        void *p = nullptr;
        int64_t rows = 0, dim = 0, stride = 0;
        at::ScalarType type = at::kFloat;
    };
    // [rows, dim] with the elements of a row side by side; `like`: of its shape and type.  `apart`: rows may lie apart.
    Rows rows(const Rows *like, bool apart, bool may_be_none = false)
    {
        Rows r;
        const at::Tensor *t = here(may_be_none);
        if (!t) return r;
        if (t->dim() != 2 || t->size(0) > INT_MAX || t->size(1) > INT_MAX) { plain = false; return r; }
        r.rows = t->size(0); r.dim = t->size(1); r.type = t->scalar_type();
        r.stride = r.rows > 1 ? t->stride(0) : r.dim;
        if ((like ? r.rows != like->rows || r.dim != like->dim || r.type != like->type : dtype(r.type) < 0) ||
            (r.rows && r.dim > 1 && t->stride(1) != 1) || (!apart && r.stride != r.dim))
            plain = false;
        else r.p = t->data_ptr();
        return r;
    }
    void *vector(int64_t n, at::ScalarType type, bool may_be_none = false)
    {
        const at::Tensor *t = here(may_be_none);
        if (!t) return nullptr;
        if (t->scalar_type() != type || !t->is_contiguous() || (n >= 0 && t->numel() != n)) { plain = false; return nullptr; }
        return t->data_ptr();
    }
    struct Heads {
        void *p = nullptr;
        int64_t rows = 0, heads = 0, dim = 0, row = 0, head = 0;
        at::ScalarType type = at::kFloat;
        bool none = false;
    };
    // [rows, heads, dim] with the elements of a head side by side; `like`: of its shape and type.
    Heads heads(const Heads *like, bool may_be_none = false)
    {
        Heads r;
        const at::Tensor *t = here(may_be_none);
        r.none = !t;
        if (!t) return r;
        if (t->dim() != 3 || t->size(0) > INT_MAX || t->size(1) > INT_MAX || t->size(2) > INT_MAX) { plain = false; return r; }
        r.rows = t->size(0); r.heads = t->size(1); r.dim = t->size(2); r.type = t->scalar_type();
        r.row = r.rows > 1 ? t->stride(0) : r.heads * r.dim;
        r.head = r.heads > 1 ? t->stride(1) : r.dim;
        if ((like ? r.rows != like->rows || r.heads != like->heads || r.dim != like->dim || r.type != like->type : dtype(r.type) < 0) ||
            (t->numel() && r.dim > 1 && t->stride(2) != 1))
            plain = false;
        else r.p = t->data_ptr();
        return r;
    }
    struct Cache {
        void *p = nullptr;
        int64_t pages = 0, heads = 0, page = 0;
    };
    // A cache [pages, heads, page, dim] for heads like `like`.
    Cache cache(const Heads &like, bool may_be_none = false)
    {
        Cache c;
        const at::Tensor *t = here(may_be_none);
        if (!t) return c;
        if (t->dim() != 4 || t->size(3) != like.dim || t->scalar_type() != like.type || !t->is_contiguous() || t->size(2) > INT_MAX ||
            t->size(1) > INT_MAX) {
            plain = false;
            return c;
        }
        c.pages = t->size(0); c.heads = t->size(1); c.page = t->size(2);
        c.p = t->data_ptr();
        return c;
    }
    void *bytes(size_t &n, bool may_be_none = false)
    {
        n = 0;
        PyObject *o = *at;
        void *p = vector(-1, at::kByte, may_be_none);
        if (plain && p) n = (size_t)THPVariable_Unpack(o).numel();
        return p;
    }
    static int dtype(at::ScalarType t) { return t == at::kFloat ? DSQ_F32 : t == at::kHalf ? DSQ_F16 : t == at::kBFloat16 ? DSQ_BF16 : -1; }
    const dsq_conv_desc *desc(dsq_conv_desc &d)
    {
        PyObject *o = *at++;
        Py_buffer view;
        if (!plain || Py_TYPE(o) != desc_type || PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            plain = false;
            return nullptr;
        }
        if (view.len == (Py_ssize_t)sizeof d) memcpy(&d, view.buf, sizeof d);
        else plain = false;
        PyBuffer_Release(&view);
        return &d;
    }
    void *stream()
    {
        PyObject *o = *at++;
        if (!plain) return nullptr;
        if (o == Py_None) return (void *)c10::hip::getCurrentHIPStream().stream();
        if (!PyLong_CheckExact(o)) { plain = false; return nullptr; }
        void *p = PyLong_AsVoidPtr(o);
        if (PyErr_Occurred()) { PyErr_Clear(); plain = false; }
        return p;
    }
};

// (a C++ exception, from a tensor without memory of its own for instance, is left to the general path)
template <class F>
PyObject *guarded(F body)
{
    try {
        return body();
    } catch (...) {
        Py_RETURN_NONE;
    }
}

template <class F>
PyObject *call(const Args &a, F f)
{
    if (!a.plain) Py_RETURN_NONE;
    dsq_status status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)status);
}

PyObject *quantize_act(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 12);
        if (!a.plain) Py_RETURN_NONE;
        const float *x = (const float *)a.tensor(at::kFloat);
        const dsq_layout layout = (dsq_layout)a.integer();
        const int N = a.integer(), C = a.integer(), H = a.integer(), W = a.integer();
        const float l = a.real(), u = a.real();
        const int bits = a.integer();
        size_t bytes = 0;
        void *codes = a.tensor(at::kByte, false, &bytes);
        int32_t *sums = (int32_t *)a.tensor(at::kInt);
        void *stream = a.stream();
        return call(a, [=] { return f_quantize_act(x, layout, N, C, H, W, l, u, bits, codes, bytes, sums, stream); });
    });
}

PyObject *conv2d(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 11);
        if (!a.plain) Py_RETURN_NONE;
        dsq_conv_desc d;
        a.desc(d);
        const void *act = a.tensor(at::kByte);
        const int32_t *sums = (const int32_t *)a.tensor(at::kInt);
        const float l = a.real(), u = a.real();
        const void *w = a.tensor(at::kByte), *aux = a.tensor(at::kByte);
        float *out = (float *)a.tensor(at::kFloat);
        const dsq_layout layout = (dsq_layout)a.integer();
        int32_t *acc = (int32_t *)a.tensor(at::kInt, true);
        void *stream = a.stream();
        return call(a, [=, &d] { return f_conv2d(&d, act, sums, l, u, w, aux, out, layout, acc, stream); });
    });
}

PyObject *conv2d_requant(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 16);
        if (!a.plain) Py_RETURN_NONE;
        dsq_conv_desc d;
        a.desc(d);
        const void *act = a.tensor(at::kByte);
        const int32_t *sums = (const int32_t *)a.tensor(at::kInt);
        const float l = a.real(), u = a.real();
        const void *w = a.tensor(at::kByte), *aux = a.tensor(at::kByte);
        const float *scale = (const float *)a.tensor(at::kFloat, true), *shift = (const float *)a.tensor(at::kFloat, true);
        const int relu = a.truth();
        const float l_next = a.real(), u_next = a.real();
        const int bits_next = a.integer();
        size_t bytes = 0;
        void *codes = a.tensor(at::kByte, false, &bytes);
        int32_t *sums_next = (int32_t *)a.tensor(at::kInt);
        void *stream = a.stream();
        return call(a, [=, &d] {
            return f_conv2d_requant(&d, act, sums, l, u, w, aux, scale, shift, relu, l_next, u_next, bits_next, codes, bytes,
                                    sums_next, stream);
        });
    });
}

PyObject *conv2d_wq(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 8);
        if (!a.plain) Py_RETURN_NONE;
        dsq_conv_desc d;
        a.desc(d);
        const float *x = (const float *)a.tensor(at::kFloat);
        const dsq_layout x_layout = (dsq_layout)a.integer();
        const void *w = a.tensor(at::kByte), *aux = a.tensor(at::kByte);
        float *out = (float *)a.tensor(at::kFloat);
        const dsq_layout out_layout = (dsq_layout)a.integer();
        void *stream = a.stream();
        return call(a, [=, &d] { return f_conv2d_wq(&d, x, x_layout, w, aux, out, out_layout, stream); });
    });
}

PyObject *soft_quantize_fwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 7);
        if (!a.plain) Py_RETURN_NONE;
        size_t count = 0;
        const float *x = (const float *)a.tensor(at::kFloat, false, &count);
        const float l = a.real(), u = a.real(), alpha = a.real();
        const int bits = a.integer();
        float *y = (float *)a.tensor(at::kFloat);
        void *stream = a.stream();
        return call(a, [=] { return f_soft_fwd(x, count, l, u, alpha, bits, y, stream); });
    });
}

PyObject *soft_quantize_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 9);
        if (!a.plain) Py_RETURN_NONE;
        size_t count = 0;
        const float *x = (const float *)a.tensor(at::kFloat, false, &count);
        const float *gy = (const float *)a.tensor(at::kFloat);
        const float l = a.real(), u = a.real(), alpha = a.real();
        const int bits = a.integer();
        float *gx = (float *)a.tensor(at::kFloat);
        double *sums = (double *)a.tensor(at::kDouble);
        void *stream = a.stream();
        return call(a, [=] { return f_soft_bwd(x, gy, count, l, u, alpha, bits, gx, sums, stream); });
    });
}

PyObject *rms_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 10);
        if (!a.plain || !f_rms_norm) Py_RETURN_NONE;
        const Args::Rows x = a.rows(nullptr, true), res = a.rows(&x, true, true);
        const void *w = a.vector(x.dim, x.type, true);
        const float eps = a.real();
        const Args::Rows sum = a.rows(&x, false, true), y = a.rows(&x, false, true);
        const Args::Rows like = {nullptr, x.rows, (int64_t)f_code_row_bytes((int)x.dim), 0, at::kChar};
        const Args::Rows codes = a.rows(&like, false, true);
        float *scales = (float *)a.vector(x.rows, at::kFloat, true), *rstd = (float *)a.vector(x.rows, at::kFloat, true);
        void *stream = a.stream();
        return call(a, [=] {
            return f_rms_norm(x.p, x.stride, res.p, res.stride, w, (dsq_dtype)Args::dtype(x.type), (int)x.rows, (int)x.dim, eps, sum.p,
                              y.p, (int8_t *)codes.p, (size_t)(codes.rows * codes.dim), scales, rstd, stream);
        });
    });
}

PyObject *rms_norm_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 9);
        if (!a.plain || !f_rms_norm_bwd) Py_RETURN_NONE;
        const Args::Rows h = a.rows(nullptr, true);
        const void *w = a.vector(h.dim, h.type, true);
        const float *rstd = (const float *)a.vector(h.rows, at::kFloat);
        const Args::Rows gy = a.rows(&h, true), gs = a.rows(&h, true, true), gx = a.rows(&h, false);
        float *gw = (float *)a.vector(h.dim, at::kFloat, true);
        size_t size;
        void *ws = a.bytes(size, true), *stream = a.stream();
        return call(a, [=] {
            return f_rms_norm_bwd(h.p, h.stride, w, rstd, gy.p, gy.stride, gs.p, gs.stride, (dsq_dtype)Args::dtype(h.type), (int)h.rows,
                                  (int)h.dim, gx.p, gw, ws, size, stream);
        });
    });
}

// w_packed, w_scales, N, K, group of a product, with the sizes of the buffers checked.
struct Layer {
    const void *w, *s;
    int N, K, group;
    explicit Layer(Args &a)
    {
        size_t wn, sn;
        w = a.bytes(wn); s = a.bytes(sn);
        N = a.integer(); K = a.integer(); group = a.integer();
        if (a.plain && (wn < f_w4_packed_bytes(N, K) || sn < f_w4_scale_bytes(N, K, group))) a.plain = false;
    }
};

PyObject *linear_w4(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 9);
        if (!a.plain || !f_linear_w4) Py_RETURN_NONE;
        const Args::Rows x = a.rows(nullptr, true);
        const Layer l(a);
        const void *bias = a.vector(l.N, x.type, true);
        const Args::Rows like = {nullptr, x.rows, l.N, 0, x.type};
        const Args::Rows out = a.rows(&like, true);
        void *stream = a.stream();
        if (x.dim != l.K) a.plain = false;
        return call(a, [=] {
            return f_linear_w4(x.p, x.stride, (dsq_dtype)Args::dtype(x.type), (int)x.rows, l.N, l.K, l.group, l.w, l.s, bias, out.p,
                               out.stride, stream);
        });
    });
}

PyObject *linear_w4a8(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 10);
        if (!a.plain || !f_linear_w4a8) Py_RETURN_NONE;
        PyObject *const *first = a.at;
        a.at = first + 8;
        const Args::Rows out = a.rows(nullptr, true);
        a.at = first;
        PyObject *const *layer = first + 2;
        if (!a.plain || !PyLong_CheckExact(layer[3])) Py_RETURN_NONE;
        const long K = PyLong_AsLong(layer[3]);
        if (K <= 0 || K > INT_MAX) { PyErr_Clear(); Py_RETURN_NONE; }
        const Args::Rows like = {nullptr, out.rows, (int64_t)f_code_row_bytes((int)K), 0, at::kChar};
        const Args::Rows q = a.rows(&like, false);
        const float *scales = (const float *)a.vector(out.rows, at::kFloat);
        const Layer l(a);
        const void *bias = a.vector(l.N, out.type, true);
        a.at = first + 9;
        void *stream = a.stream();
        if (out.dim != l.N) a.plain = false;
        return call(a, [=] {
            return f_linear_w4a8((const int8_t *)q.p, (size_t)(q.rows * q.dim), scales, (int)out.rows, l.N, l.K, l.group, l.w, l.s, bias,
                                 (dsq_dtype)Args::dtype(out.type), out.p, out.stride, stream);
        });
    });
}

// positions [rows] or [axes, rows], pair_axis, frequencies, interleaved
struct Rotation {
    const int32_t *positions;
    const uint8_t *pair_axis;
    const float *frequencies;
    int axes = 1, rope_dim = 0, interleaved;
    Rotation(Args &a, int64_t rows)
    {
        PyObject *o = a.at[0], *f = a.at[2];
        const auto tensor = [](PyObject *x) { return THPVariable_CheckTypeExact(Py_TYPE(x)) && THPVariable_Unpack(x).defined(); };
        if (tensor(o) && THPVariable_Unpack(o).dim() == 2) axes = (int)std::min<int64_t>(THPVariable_Unpack(o).size(0), INT_MAX);
        int64_t pairs = 0;
        if (tensor(f)) pairs = THPVariable_Unpack(f).numel();
        if (pairs > INT_MAX / 2) a.plain = false;
        positions = (const int32_t *)a.vector(axes * rows, at::kInt, true);
        pair_axis = (const uint8_t *)a.vector(pairs, at::kByte, true);
        frequencies = (const float *)a.vector(pairs, at::kFloat, true);
        rope_dim = (int)(2 * pairs);
        interleaved = a.truth();
    }
};

PyObject *qk_norm_rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 16);
        if (!a.plain || !f_qk_norm_rope) Py_RETURN_NONE;
        const Args::Heads q = a.heads(nullptr), k = a.heads(nullptr), v = a.heads(&k, true);
        const void *qw = a.vector(q.dim, q.type, true), *kw = a.vector(q.dim, q.type, true);
        const float eps = a.real();
        const Rotation r(a, q.rows);
        const Args::Heads qo = a.heads(&q), ko = a.heads(&k, true);
        const Args::Cache kc = a.cache(k, true), vc = a.cache(k, true);
        const int64_t *slots = (const int64_t *)a.vector(q.rows, at::kLong, true);
        void *stream = a.stream();
        if (k.rows != q.rows || k.dim != q.dim || k.type != q.type || kc.pages != vc.pages || kc.page != vc.page ||
            ((kc.p || vc.p) && (kc.heads != k.heads || vc.heads != k.heads)) || ((vc.p || slots) && !kc.p))
            a.plain = false;
        return call(a, [=] {
            return f_qk_norm_rope(q.p, q.row, q.head, k.p, k.row, k.head, v.p, v.row, v.head, (dsq_dtype)Args::dtype(q.type), (int)q.rows,
                                  (int)q.heads, (int)k.heads, (int)q.dim, qw, kw, eps, r.positions, r.axes, r.pair_axis, r.frequencies,
                                  r.rope_dim, r.interleaved, qo.p, qo.row, qo.head, ko.p, ko.row, ko.head, kc.p, vc.p, kc.pages,
                                  (int)kc.page, slots, stream);
        });
    });
}

PyObject *qk_norm_rope_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 17);
        if (!a.plain || !f_qk_norm_rope_bwd) Py_RETURN_NONE;
        const Args::Heads q = a.heads(nullptr), k = a.heads(nullptr);
        const void *qw = a.vector(q.dim, q.type, true), *kw = a.vector(q.dim, q.type, true);
        const float eps = a.real();
        const Rotation r(a, q.rows);
        const Args::Heads gqo = a.heads(&q), gko = a.heads(&k), gq = a.heads(&q), gk = a.heads(&k);
        float *gqw = (float *)a.vector(q.dim, at::kFloat, true), *gkw = (float *)a.vector(q.dim, at::kFloat, true);
        size_t size;
        void *ws = a.bytes(size, true), *stream = a.stream();
        if (k.rows != q.rows || k.dim != q.dim || k.type != q.type) a.plain = false;
        return call(a, [=] {
            return f_qk_norm_rope_bwd(q.p, q.row, q.head, k.p, k.row, k.head, (dsq_dtype)Args::dtype(q.type), (int)q.rows, (int)q.heads,
                                      (int)k.heads, (int)q.dim, qw, kw, eps, r.positions, r.axes, r.pair_axis, r.frequencies, r.rope_dim,
                                      r.interleaved, gqo.p, gqo.row, gqo.head, gko.p, gko.row, gko.head, gq.p, gq.row, gq.head, gk.p, gk.row,
                                      gk.head, gqw, gkw, ws, size, stream);
        });
    });
}

// q_starts and k_starts, either of which may be None.
struct Starts {
    const int32_t *q, *k;
    int64_t sequences = 1;
    explicit Starts(Args &a)
    {
        PyObject *o = a.at[0];
        if (a.plain && o != Py_None && THPVariable_CheckTypeExact(Py_TYPE(o)) && THPVariable_Unpack(o).defined())
            sequences = THPVariable_Unpack(o).numel() - 1;
        if (sequences < 0 || sequences > INT_MAX) a.plain = false;
        q = (const int32_t *)a.vector(sequences + 1, at::kInt, true);
        k = (const int32_t *)a.vector(sequences + 1, at::kInt, true);
    }
};

PyObject *attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 10);
        if (!a.plain || !f_attention) Py_RETURN_NONE;
        const Args::Heads q = a.heads(nullptr), k = a.heads(nullptr), v = a.heads(&k);
        const Starts s(a);
        const int causal = a.truth();
        const float scale = a.real();
        const Args::Heads out = a.heads(&q);
        float *lse = (float *)a.vector(q.heads * q.rows, at::kFloat, true);
        void *stream = a.stream();
        if (k.dim != q.dim || k.type != q.type) a.plain = false;
        return call(a, [=] {
            return f_attention(q.p, q.row, q.head, k.p, k.row, k.head, v.p, v.row, v.head, (dsq_dtype)Args::dtype(q.type), (int)q.rows,
                               (int)k.rows, (int)q.heads, (int)k.heads, (int)q.dim, s.q, s.k, (int)s.sequences, causal, scale, out.p, out.row,
                               out.head, lse, stream);
        });
    });
}

PyObject *attention_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 15);
        if (!a.plain || !f_attention_bwd) Py_RETURN_NONE;
        const Args::Heads q = a.heads(nullptr), k = a.heads(nullptr), v = a.heads(&k), out = a.heads(&q);
        const float *lse = (const float *)a.vector(q.heads * q.rows, at::kFloat);
        const Args::Heads go = a.heads(&q);
        const Starts s(a);
        const int causal = a.truth();
        const float scale = a.real();
        const Args::Heads gq = a.heads(&q), gk = a.heads(&k), gv = a.heads(&k);
        size_t size;
        void *ws = a.bytes(size, true), *stream = a.stream();
        if (k.dim != q.dim || k.type != q.type) a.plain = false;
        return call(a, [=] {
            return f_attention_bwd(q.p, q.row, q.head, k.p, k.row, k.head, v.p, v.row, v.head, out.p, out.row, out.head, lse, go.p, go.row,
                                   go.head, (dsq_dtype)Args::dtype(q.type), (int)q.rows, (int)k.rows, (int)q.heads, (int)k.heads, (int)q.dim,
                                   s.q, s.k, (int)s.sequences, causal, scale, gq.p, gq.row, gq.head, gk.p, gk.row, gk.head, gv.p, gv.row,
                                   gv.head, ws, size, stream);
        });
    });
}

PyObject *attention_cache(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Args a(args, n, 12);
        if (!a.plain || !f_attention_cache) Py_RETURN_NONE;
        const Args::Heads q = a.heads(nullptr);
        PyObject *o = args[6];                                               // lengths
        if (!THPVariable_CheckTypeExact(Py_TYPE(o)) || !THPVariable_Unpack(o).defined()) Py_RETURN_NONE;
        const int64_t sequences = THPVariable_Unpack(o).numel();
        if (sequences > INT_MAX) Py_RETURN_NONE;
        const int32_t *starts = (const int32_t *)a.vector(sequences + 1, at::kInt, true);
        const int max_rows = a.integer();
        const Args::Cache kc = a.cache(q), vc = a.cache(q);
        Args::Rows table;
        if (const at::Tensor *t = a.here(false)) {
            if (t->dim() != 2 || t->size(0) != sequences || t->size(1) > INT_MAX || t->scalar_type() != at::kInt ||
                (t->numel() && t->size(1) > 1 && t->stride(1) != 1))
                a.plain = false;
            else {
                table.p = t->data_ptr();
                table.dim = t->size(1);
                table.stride = sequences > 1 ? t->stride(0) : table.dim;
            }
        }
        const int32_t *lengths = (const int32_t *)a.vector(sequences, at::kInt);
        int64_t words = 0;
        o = *a.at;
        if (o != Py_None) {
            if (!a.plain || !THPVariable_CheckTypeExact(Py_TYPE(o)) || !THPVariable_Unpack(o).defined() || THPVariable_Unpack(o).dim() != 2) Py_RETURN_NONE;
            words = THPVariable_Unpack(o).size(1);
            if (words <= 0 || words > INT_MAX) Py_RETURN_NONE;
        }
        const uint64_t *tree = (const uint64_t *)a.vector(q.rows * words, at::kLong, true);
        const float scale = a.real();
        const Args::Heads out = a.heads(&q);
        size_t size;
        void *ws = a.bytes(size), *stream = a.stream();
        if (kc.heads != vc.heads || kc.pages != vc.pages || kc.page != vc.page) a.plain = false;
        return call(a, [=] {
            return f_attention_cache(q.p, q.row, q.head, (dsq_dtype)Args::dtype(q.type), (int)q.rows, (int)q.heads, (int)kc.heads, (int)q.dim,
                                     starts, (int)sequences, max_rows, kc.p, vc.p, kc.pages, (int)kc.page, (const int32_t *)table.p,
                                     table.stride, (int)table.dim, lengths, tree, (int)words, scale, out.p, out.row, out.head, ws, size, stream);
        });
    });
}

// init_heads(addresses of the calls for heads, in the order below)
PyObject *init_heads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "init_heads(five addresses)");
        return nullptr;
    }
    void *p[5];
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    f_qk_norm_rope = (decltype(f_qk_norm_rope))p[0];
    f_qk_norm_rope_bwd = (decltype(f_qk_norm_rope_bwd))p[1];
    f_attention = (decltype(f_attention))p[2];
    f_attention_bwd = (decltype(f_attention_bwd))p[3];
    f_attention_cache = (decltype(f_attention_cache))p[4];
    Py_RETURN_NONE;
}

// init_lm(addresses of the calls for language-model layers and their size queries, in the order below)
PyObject *init_lm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "init_lm(seven addresses)");
        return nullptr;
    }
    void *p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    f_rms_norm = (decltype(f_rms_norm))p[0];
    f_rms_norm_bwd = (decltype(f_rms_norm_bwd))p[1];
    f_linear_w4 = (decltype(f_linear_w4))p[2];
    f_linear_w4a8 = (decltype(f_linear_w4a8))p[3];
    f_code_row_bytes = (decltype(f_code_row_bytes))p[4];
    f_w4_packed_bytes = (decltype(f_w4_packed_bytes))p[5];
    f_w4_scale_bytes = (decltype(f_w4_scale_bytes))p[6];
    Py_RETURN_NONE;
}

// init(desc_type, addresses of the six entry points, in the order below)
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7 || !PyType_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "init(desc_type, six addresses)");
        return nullptr;
    }
    void *p[6];
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(args[1 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XDECREF((PyObject *)desc_type);
    desc_type = (PyTypeObject *)args[0];
    f_conv2d = (decltype(f_conv2d))p[1];
    f_conv2d_requant = (decltype(f_conv2d_requant))p[2];
    f_conv2d_wq = (decltype(f_conv2d_wq))p[3];
    f_soft_fwd = (decltype(f_soft_fwd))p[4];
    f_soft_bwd = (decltype(f_soft_bwd))p[5];
    f_quantize_act = (decltype(f_quantize_act))p[0];
    Py_RETURN_NONE;
}

#define METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(init), METHOD(quantize_act), METHOD(conv2d), METHOD(conv2d_requant), METHOD(conv2d_wq),
                         METHOD(soft_quantize_fwd), METHOD(soft_quantize_bwd), METHOD(init_lm), METHOD(rms_norm),
                         METHOD(rms_norm_bwd), METHOD(linear_w4), METHOD(linear_w4a8), METHOD(init_heads), METHOD(qk_norm_rope),
                         METHOD(qk_norm_rope_bwd), METHOD(attention), METHOD(attention_bwd), METHOD(attention_cache), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module_def); }
