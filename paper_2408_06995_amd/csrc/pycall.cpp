// The calls of the binding that programs make per layer and step, as a CPython extension (_fpqcall): argument
// marshalling only, as in binding.py, without ctypes.
//
// A layer call of a small layer costs what the host needs to make it.  Through ctypes the marshalling took 5.5 us per
// call (2.9 of them torch.cuda.current_stream(), the rest one wrapper object per argument) next to 3.5 us for the C call
// with its launch; here it takes under 1 us: tensors give their address through data_ptr(), the stream comes from the raw
// stream query.  Arguments, names and defaults are those of the Python functions that this replaces; the functions of
// libfpq.so are looked up once through the resolver that binding.py registers, and a status other than FPQ_OK goes to its
// checker, which raises FpqError.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <string.h>
#include <type_traits>

#include "../../include/fpq.h"

namespace {

PyObject* g_resolve = nullptr;      // resolver(name) -> address of the C function
PyObject* g_check = nullptr;        // checker(status, name): raises
PyObject *g_format = nullptr, *g_problem = nullptr, *g_array = nullptr;   // fpq_format_t, fpq_gemm_problem_t, ctypes.Array
PyObject *s_type, *s_data_ptr, *s_numel, *s_element_size, *s_shape, *s_stride, *s_dtype, *s_is_contiguous;
PyObject *g_float32 = nullptr, *g_bfloat16 = nullptr, *g_int32 = nullptr;
PyObject *g_get_device = nullptr, *g_get_stream = nullptr;

constexpr int kBad = 1;             // a Python error is set (statuses of the library are <= 0)

struct Args {
    PyObject* const* a;
    bool bad = false;

    // (after a failure the remaining arguments are not looked at: the first error is the one reported)
    long long integer(int i)
    {
        if (bad) return 0;
        PyObject* o = a[i];
        if (PyLong_CheckExact(o)) {
            const long long v = PyLong_AsLongLong(o);
            if (v == -1 && PyErr_Occurred()) bad = true;
            return v;
        }
        PyObject* n = PyNumber_Long(o);
        if (!n) { bad = true; return 0; }
        const long long v = PyLong_AsLongLong(n);
        Py_DECREF(n);
        if (v == -1 && PyErr_Occurred()) bad = true;
        return v;
    }
    int i(int k) { return (int)integer(k); }
    // a size: whole numbers only, no conversion
    int64_t l(int k)
    {
        if (bad) return 0;
        if (!PyLong_Check(a[k])) {
            PyErr_Format(PyExc_TypeError, "sizes are ints, not %s", Py_TYPE(a[k])->tp_name);
            bad = true;
            return 0;
        }
        return (int64_t)integer(k);
    }
    int d(int k) { return (int)l(k); }
    float f(int k)
    {
        if (bad) return 0.0f;
        const double v = PyFloat_AsDouble(a[k]);
        if (v == -1.0 && PyErr_Occurred()) bad = true;
        return (float)v;
    }
    double real(int k)
    {
        if (bad) return 0.0;
        const double v = PyFloat_AsDouble(a[k]);
        if (v == -1.0 && PyErr_Occurred()) bad = true;
        return v;
    }
    // data_ptr() of a tensor; None: null
    void* ptr_of(PyObject* o)
    {
        if (bad || o == Py_None) return nullptr;
        PyObject* r = PyObject_CallMethodNoArgs(o, s_data_ptr);
        if (!r) { bad = true; return nullptr; }
        void* p = PyLong_AsVoidPtr(r);
        Py_DECREF(r);
        if (!p && PyErr_Occurred()) bad = true;
        return p;
    }
    void* p(int k) { return ptr_of(a[k]); }
    float* fp(int k) { return static_cast<float*>(p(k)); }
    uint8_t* bp(int k) { return static_cast<uint8_t*>(p(k)); }
    size_t method(PyObject* o, PyObject* name)
    {
        if (bad) return 0;
        PyObject* r = PyObject_CallMethodNoArgs(o, name);
        if (!r) { bad = true; return 0; }
        const size_t v = PyLong_AsSize_t(r);
        Py_DECREF(r);
        if (v == (size_t)-1 && PyErr_Occurred()) bad = true;
        return v;
    }
    size_t numel(int k) { return method(a[k], s_numel); }
    size_t bytes(int k) { return a[k] == Py_None ? 0 : method(a[k], s_numel) * method(a[k], s_element_size); }
    // dimension `dim` of a tensor that must have `ndim` (0: any number)
    int64_t size(int k, int dim, int ndim)
    {
        if (bad) return 0;
        PyObject* sh = PyObject_GetAttr(a[k], s_shape);
        if (!sh) { bad = true; return 0; }
        const Py_ssize_t have = PySequence_Size(sh);
        if (have < 0 || (ndim && have != ndim)) {
            if (have >= 0) PyErr_Format(PyExc_ValueError, "a tensor of %d dimensions expected, not %zd", ndim, have);
            Py_DECREF(sh);
            bad = true;
            return 0;
        }
        PyObject* d = PySequence_GetItem(sh, dim);
        Py_DECREF(sh);
        if (!d) { bad = true; return 0; }
        const long long v = PyLong_AsLongLong(d);
        Py_DECREF(d);
        if (v == -1 && PyErr_Occurred()) bad = true;
        return v;
    }
    // shape and strides of a tensor that must have `ndim` dimensions, the elements of the last one neighbours
    void layout(int k, int ndim, int64_t* size, int64_t* stride, const char* name)
    {
        if (bad) return;
        PyObject* sh = PyObject_GetAttr(a[k], s_shape);
        PyObject* st = sh ? PyObject_CallMethodNoArgs(a[k], s_stride) : nullptr;
        if (!st) { Py_XDECREF(sh); bad = true; return; }
        if (PySequence_Size(sh) != ndim || PySequence_Size(st) != ndim) {
            PyErr_Format(PyExc_ValueError, "%s: a tensor of %d dimensions expected", name, ndim);
            bad = true;
        }
        for (int d = 0; d < ndim && !bad; ++d) {
            PyObject* n = PySequence_GetItem(sh, d);
            PyObject* m = n ? PySequence_GetItem(st, d) : nullptr;
            if (m) {
                size[d] = PyLong_AsLongLong(n);
                stride[d] = PyLong_AsLongLong(m);
            }
            bad = !m || PyErr_Occurred();
            Py_XDECREF(n);
            Py_XDECREF(m);
        }
        Py_DECREF(sh);
        Py_DECREF(st);
        if (!bad && size[ndim - 1] > 1 && stride[ndim - 1] != 1) {
            PyErr_Format(PyExc_ValueError, "%s: the elements of the last dimension are not neighbours", name);
            bad = true;
        }
    }
    // the dtype of a tensor, a new reference, and torch's own to compare it with
    PyObject* dtype(int k)
    {
        if (!g_float32) {
            PyObject* m = PyImport_ImportModule("torch");
            if (!m) { bad = true; return nullptr; }
            g_float32 = PyObject_GetAttrString(m, "float32");
            g_bfloat16 = PyObject_GetAttrString(m, "bfloat16");
            g_int32 = PyObject_GetAttrString(m, "int32");
            Py_DECREF(m);
            if (!g_float32 || !g_bfloat16 || !g_int32) { Py_CLEAR(g_float32); bad = true; return nullptr; }
        }
        PyObject* t = PyObject_GetAttr(a[k], s_dtype);
        if (!t) bad = true;
        return t;
    }
    // fpq_type of a tensor
    int type(int k, const char* name)
    {
        if (bad) return 0;
        PyObject* t = dtype(k);
        if (!t) return 0;
        const int r = t == g_float32 ? FPQ_TYPE_FP32 : t == g_bfloat16 ? FPQ_TYPE_BF16 : -1;
        if (r < 0) {
            PyErr_Format(PyExc_TypeError, "%s: float32 or bfloat16 expected, not %S", name, t);
            bad = true;
        }
        Py_DECREF(t);
        return r;
    }
    void same(bool ok, const char* what)
    {
        if (bad || ok) return;
        PyErr_SetString(PyExc_ValueError, what);
        bad = true;
    }
    // elements of a contiguous tensor of P (float or int32_t), given as None or with exactly n
    template <typename P>
    P* words(int k, int64_t n, const char* name)
    {
        if (bad || a[k] == Py_None) return nullptr;
        if (method(a[k], s_numel) != (size_t)n || method(a[k], s_element_size) != 4) {
            if (!bad) PyErr_Format(PyExc_ValueError, "%s: %lld elements of four bytes expected", name, (long long)n);
            bad = true;
            return nullptr;
        }
        PyObject* t = dtype(k);
        if (!t) return nullptr;
        const bool whole = std::is_same<typename std::remove_const<P>::type, int32_t>::value;
        if (t != (whole ? g_int32 : g_float32)) {
            PyErr_Format(PyExc_TypeError, "%s: %s expected, not %S", name, whole ? "int32" : "float32", t);
            bad = true;
        }
        Py_DECREF(t);
        if (bad) return nullptr;
        PyObject* c = PyObject_CallMethodNoArgs(a[k], s_is_contiguous);
        if (!c || c != Py_True) {
            if (c) PyErr_Format(PyExc_ValueError, "%s: not contiguous", name);
            bad = true;
        }
        Py_XDECREF(c);
        return static_cast<P*>(p(k));
    }
    // the ctypes structure, or anything with four elements (e, m, b, c)
    fpq_format_t fmt(int k)
    {
        fpq_format_t r;
        memset(&r, 0, sizeof r);
        if (bad) return r;
        PyObject* o = a[k];
        if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 4) {
            Args t{&PyTuple_GET_ITEM(o, 0)};
            r.ebits = t.i(0); r.mbits = t.i(1); r.bias = t.i(2); r.maxval = t.f(3);
            bad |= t.bad;
            return r;
        }
        const int is = PyObject_IsInstance(o, g_format);
        if (is < 0) { bad = true; return r; }
        if (is) {
            Py_buffer b;
            if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) { bad = true; return r; }
            memcpy(&r, b.buf, sizeof r);
            PyBuffer_Release(&b);
            return r;
        }
        PyObject* t = PySequence_Tuple(o);
        if (!t) { bad = true; return r; }
        if (PyTuple_GET_SIZE(t) == 4) {
            Args u{&PyTuple_GET_ITEM(t, 0)};
            r.ebits = u.i(0); r.mbits = u.i(1); r.bias = u.i(2); r.maxval = u.f(3);
            bad |= u.bad;
        } else {
            PyErr_SetString(PyExc_TypeError, "a format is (e, m, b, c)");
            bad = true;
        }
        Py_DECREF(t);
        return r;
    }
    // the current torch stream of the current device
    void* stream()
    {
        if (bad) return nullptr;
        if (!g_get_stream) {
            PyObject* m = PyImport_ImportModule("torch._C");
            if (!m) { bad = true; return nullptr; }
            g_get_device = PyObject_GetAttrString(m, "_cuda_getDevice");
            g_get_stream = PyObject_GetAttrString(m, "_cuda_getCurrentRawStream");
            Py_DECREF(m);
            if (!g_get_device || !g_get_stream) { Py_CLEAR(g_get_stream); bad = true; return nullptr; }
        }
        PyObject* d = PyObject_CallNoArgs(g_get_device);
        if (!d) { bad = true; return nullptr; }
        PyObject* r = PyObject_CallOneArg(g_get_stream, d);
        Py_DECREF(d);
        if (!r) { bad = true; return nullptr; }
        void* p = PyLong_AsVoidPtr(r);
        Py_DECREF(r);
        if (!p && PyErr_Occurred()) bad = true;
        return p;
    }
};

template <typename F>
F resolve(F, const char* name)
{
    PyObject* r = g_resolve ? PyObject_CallFunction(g_resolve, "s", name) : nullptr;
    if (!r) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "_fpqcall is not set up");
        return nullptr;
    }
    void* p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return reinterpret_cast<F>(p);
}

// Calls the library with the interpreter released, as ctypes does (a full queue makes a launch wait).
template <typename F, typename... V>
int invoke(const Args& A, F fn, V... v)
{
    if (A.bad) return kBad;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = fn(v...);
    Py_END_ALLOW_THREADS
    return st;
}

#define FN(name)                                     \
    static decltype(&name) fn = nullptr;             \
    if (!fn && !(fn = resolve(&name, #name))) return kBad

// a: arguments in order, missing trailing ones replaced by their defaults
int do_gemm(Args& A)
{
    FN(fpq_gemm);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fp(9), A.l(10), A.l(11),
                  A.l(12), A.i(13), A.p(14), A.bytes(14), A.stream());
}
int do_gemm_noalloc(Args& A)
{
    FN(fpq_gemm_noalloc);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fp(9), A.l(10), A.l(11),
                  A.l(12), A.i(13), A.stream());
}
int do_conv2d(Args& A)
{
    FN(fpq_conv2d);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fp(9), A.l(10), A.l(11),
                  A.l(12), A.l(13), A.l(14), A.d(15), A.d(16), A.d(17), A.d(18), A.i(19), A.p(20), A.bytes(20), A.stream());
}
int do_gemm_codes_out(Args& A)
{
    FN(fpq_gemm_codes_out);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fmt(9), A.f(10), A.fp(11),
                  A.bp(12), A.l(13), A.l(14), A.l(15), A.i(16), A.p(17), A.bytes(17), A.stream());
}
int do_conv2d_codes_out(Args& A)
{
    FN(fpq_conv2d_codes_out);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fmt(9), A.f(10), A.fp(11),
                  A.bp(12), A.l(13), A.l(14), A.l(15), A.l(16), A.l(17), A.d(18), A.d(19), A.d(20), A.d(21), A.i(22), A.p(23),
                  A.bytes(23), A.stream());
}
int do_gemm_sparse(Args& A)
{
    FN(fpq_gemm_sparse);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fp(9), A.l(10), A.l(11),
                  A.l(12), A.p(13), A.bytes(13), A.stream());
}
int do_conv2d_sparse(Args& A)
{
    FN(fpq_conv2d_sparse);
    return invoke(A, fn, A.p(0), A.i(1), A.fmt(2), A.f(3), A.fp(4), A.p(5), A.fmt(6), A.fp(7), A.fp(8), A.fp(9), A.l(10), A.l(11),
                  A.l(12), A.l(13), A.l(14), A.d(15), A.d(16), A.d(17), A.d(18), A.p(19), A.bytes(19), A.stream());
}
int do_gemm_grouped(Args& A)
{
    FN(fpq_gemm_grouped);
    // the array of gemm_problems() and nothing else that has a buffer: the library reads addresses from it
    PyObject* of = PyObject_IsInstance(A.a[0], g_array) == 1 ? PyObject_GetAttr(A.a[0], s_type) : nullptr;
    const bool problems = of == g_problem;
    Py_XDECREF(of);
    if (!problems) {
        if (!PyErr_Occurred()) PyErr_Format(PyExc_TypeError, "problems: the array of gemm_problems(), not %s", Py_TYPE(A.a[0])->tp_name);
        return kBad;
    }
    Py_buffer b;
    if (PyObject_GetBuffer(A.a[0], &b, PyBUF_SIMPLE)) return kBad;
    const int st = invoke(A, fn, static_cast<const fpq_gemm_problem_t*>(b.buf), (int)(b.len / (Py_ssize_t)sizeof(fpq_gemm_problem_t)),
                          A.i(1), A.fmt(2), A.fmt(3), A.i(4), A.p(5), A.bytes(5), A.stream());
    PyBuffer_Release(&b);
    return st;
}
int do_absmax(Args& A)
{
    FN(fpq_absmax);
    return invoke(A, fn, A.fp(0), A.numel(0), A.f(1), A.fp(2), A.fp(3), A.p(4), A.bytes(4), A.stream());
}
int do_quantize(Args& A)
{
    FN(fpq_quantize);
    return invoke(A, fn, A.fp(0), A.numel(0), A.fmt(1), A.f(2), A.fp(3), A.bp(4), A.stream());
}
int do_quantize_nhwc(Args& A)
{
    FN(fpq_quantize_nhwc);
    return invoke(A, fn, A.fp(0), A.size(0, 0, 4), A.size(0, 1, 4), A.size(0, 2, 4), A.size(0, 3, 4),
                  A.fmt(1), A.f(2), A.fp(3), A.bp(4), A.stream());
}
int do_int_calibrate(Args& A)
{
    FN(fpq_int_calibrate);
    return invoke(A, fn, A.fp(0), A.numel(0), A.i(1), static_cast<fpq_int_params*>(A.p(2)), A.p(3), A.bytes(3), A.stream());
}
int do_int_quantize(Args& A)
{
    FN(fpq_int_quantize);
    return invoke(A, fn, A.fp(0), A.numel(0), A.i(1), A.f(2), (int32_t)A.i(3), static_cast<const fpq_int_params*>(A.p(4)), A.bp(5),
                  A.stream());
}
int do_int_gemm(Args& A)
{
    FN(fpq_int_gemm);
    return invoke(A, fn, A.bp(0), A.f(1), (int32_t)A.i(2), static_cast<const fpq_int_params*>(A.p(3)), A.p(4), A.i(5), A.fp(6),
                  static_cast<const int32_t*>(A.p(7)), A.fp(8), A.fp(9), A.l(10), A.l(11), A.l(12), A.p(13), A.bytes(13), A.stream());
}
int do_rl_step(Args& A)
{
    FN(fpq_rl_step);
    return invoke(A, fn, A.fp(0), A.fp(1), A.size(0, 0, 2), A.size(0, 1, 2), A.fmt(2), A.fp(3), A.fp(4), A.size(4, 0, 0), A.f(5), A.f(6), A.fp(7),
                  A.fp(8), A.p(9), A.bytes(9), A.stream());
}
int do_search_format(Args& A)
{
    FN(fpq_search_format);
    int32_t e[64], m[64];                        // the library takes at most 8 and says so
    int n = 0;
    PyObject* seq = PySequence_Fast(A.a[1], "encodings: a sequence of (e, m)");
    if (!seq) return kBad;
    const Py_ssize_t len = PySequence_Fast_GET_SIZE(seq);
    for (Py_ssize_t k = 0; k < len && k < 64 && !A.bad; ++k, ++n) {
        PyObject* t = PySequence_Tuple(PySequence_Fast_GET_ITEM(seq, k));
        if (!t || PyTuple_GET_SIZE(t) != 2) {
            if (t) PyErr_SetString(PyExc_ValueError, "encodings: a sequence of (e, m)");
            A.bad = true;
        } else {
            Args u{&PyTuple_GET_ITEM(t, 0)};
            e[k] = u.i(0);
            m[k] = u.i(1);
            A.bad |= u.bad;
        }
        Py_XDECREF(t);
    }
    Py_DECREF(seq);
    return invoke(A, fn, A.fp(0), A.numel(0), (const int32_t*)e, (const int32_t*)m, n, A.i(2), A.fp(3),
                  static_cast<fpq_search_result*>(A.p(4)), A.p(5), A.bytes(5), A.stream());
}

// [batch, tokens, heads, dim] tensors: sizes, strides and type, which all must agree
fpq_attention_args_t attention_args(Args& A, int scale, int causal, int lens)
{
    fpq_attention_args_t r;
    memset(&r, 0, sizeof r);
    int64_t q[4], k[4], v[4], o[4], s[4];
    A.layout(0, 4, q, s, "q");
    memcpy(r.q_strides, s, sizeof r.q_strides);
    A.layout(1, 4, k, s, "k");
    memcpy(r.k_strides, s, sizeof r.k_strides);
    A.layout(2, 4, v, s, "v");
    memcpy(r.v_strides, s, sizeof r.v_strides);
    A.layout(3, 4, o, s, "o");
    memcpy(r.o_strides, s, sizeof r.o_strides);
    r.type = A.type(0, "q");
    if (A.bad) return r;
    A.same(A.type(1, "k") == r.type && A.type(2, "v") == r.type && A.type(3, "o") == r.type, "q, k, v and o of one type expected");
    A.same(!memcmp(q, o, sizeof q), "o: the shape of q expected");
    A.same(!memcmp(k, v, sizeof k), "v: the shape of k expected");
    A.same(q[0] == k[0] && q[3] == k[3], "k: the samples and the head dimension of q expected");
    if (A.bad) return r;
    r.batch = q[0];
    r.q_len = q[1];
    r.q_heads = q[2];
    r.head_dim = q[3];
    r.kv_len = k[1];
    r.kv_heads = k[2];
    r.scale = A.f(scale);
    r.causal = A.i(causal);
    r.kv_lens = A.words<const int32_t>(lens, r.batch, "kv_lens");
    return r;
}
int do_attention(Args& A)
{
    FN(fpq_attention);
    const fpq_attention_args_t r = attention_args(A, 5, 6, 7);
    float* const lse = A.words<float>(4, r.batch * r.q_heads * r.q_len, "lse");
    return invoke(A, fn, &r, A.p(0), A.p(1), A.p(2), A.p(3), lse, A.p(8), A.bytes(8), A.stream());
}
int do_attention_backward(Args& A)
{
    FN(fpq_attention_backward);
    fpq_attention_args_t r = attention_args(A, 9, 10, 11);
    static const char* const names[4] = {"grad_o", "grad_q", "grad_k", "grad_v"};
    int64_t* const strides[4] = {r.grad_o_strides, r.grad_q_strides, r.grad_k_strides, r.grad_v_strides};
    for (int t = 0; t < 4 && !A.bad; ++t) {
        int64_t n[4], s[4];
        A.layout(5 + t, 4, n, s, names[t]);
        memcpy(strides[t], s, sizeof r.grad_o_strides);
        A.same(A.type(5 + t, names[t]) == r.type, "gradients: the type of q expected");
        if (A.bad) break;
        const int64_t len = t < 2 ? r.q_len : r.kv_len, heads = t < 2 ? r.q_heads : r.kv_heads;
        A.same(n[0] == r.batch && n[1] == len && n[2] == heads && n[3] == r.head_dim, "gradients: the shapes of o, q, k and v expected");
    }
    const float* const lse = A.words<const float>(4, r.batch * r.q_heads * r.q_len, "lse");
    return invoke(A, fn, &r, A.p(0), A.p(1), A.p(2), A.p(3), lse, A.p(5), A.p(6), A.p(7), A.p(8), A.p(12), A.bytes(12), A.stream());
}

// x, a, b, scaling, row_start, adapter: the first six arguments of both calls
fpq_adapter_args_t adapter_args(Args& A)
{
    fpq_adapter_args_t r;
    memset(&r, 0, sizeof r);
    int64_t x[2] = {}, sx[2] = {}, a[3] = {}, b[3] = {}, s[3] = {}, q[1] = {};
    A.layout(0, 2, x, sx, "x");
    A.layout(1, 3, a, s, "a");
    if (!A.bad) A.same(s[1] == a[2] || a[1] <= 1, "a: not contiguous");
    if (!A.bad) A.same(s[0] == a[1] * a[2] || a[0] <= 1, "a: not contiguous");
    A.layout(2, 3, b, s, "b");
    if (!A.bad) A.same(s[1] == b[2] || b[1] <= 1, "b: not contiguous");
    if (!A.bad) A.same(s[0] == b[1] * b[2] || b[0] <= 1, "b: not contiguous");
    A.layout(5, 1, q, s, "adapter");
    r.x_type = A.type(0, "x");
    r.w_type = A.type(1, "a");
    if (A.bad) return r;
    A.same(A.type(2, "b") == r.w_type, "a and b of one type expected");
    A.same(a[0] == b[0] && a[1] == b[2], "a [adapters, R, K] and b [adapters, N, R] expected");
    A.same(x[1] == a[2], "x: rows of the adapters' K expected");
    r.M = x[0];
    r.K = x[1];
    r.R = a[1];
    r.N = b[1];
    r.adapters = a[0];
    r.requests = q[0];
    r.ld_x = x[0] > 1 ? sx[0] : x[1];
    r.scaling = A.words<const float>(3, r.adapters, "scaling");
    r.row_start = A.words<const int32_t>(4, r.requests + 1, "row_start");
    r.adapter = A.words<const int32_t>(5, r.requests, "adapter");
    return r;
}
// A matrix of `rows` x `cols` of x's type, or None: its row stride
int64_t adapter_rows(Args& A, int k, const fpq_adapter_args_t& r, int64_t cols, const char* name)
{
    if (A.bad || A.a[k] == Py_None) return cols;
    int64_t n[2], s[2];
    A.layout(k, 2, n, s, name);
    if (A.bad) return 0;
    if (n[0] != r.M || n[1] != cols || A.type(k, name) != r.x_type) {
        if (!A.bad) PyErr_Format(PyExc_ValueError, "%s: rows of x, %lld columns and the type of x expected", name, (long long)cols);
        A.bad = true;
    }
    return n[0] > 1 ? s[0] : cols;
}
int do_adapter_apply(Args& A)
{
    FN(fpq_adapter_apply);
    fpq_adapter_args_t r = adapter_args(A);
    r.ld_base = adapter_rows(A, 6, r, r.N, "base");
    r.ld_y = adapter_rows(A, 7, r, r.N, "y");
    float* const t = A.words<float>(8, r.M * r.R, "t");
    return invoke(A, fn, &r, A.p(0), A.p(1), A.p(2), A.p(6), A.p(7), t, A.p(9), A.bytes(9), A.stream());
}
int do_adapter_backward(Args& A)
{
    FN(fpq_adapter_backward);
    fpq_adapter_args_t r = adapter_args(A);
    const float* const t = A.words<const float>(6, r.M * r.R, "t");
    r.ld_grad_y = adapter_rows(A, 7, r, r.N, "grad_y");
    r.ld_grad_x_base = adapter_rows(A, 8, r, r.K, "grad_x_base");
    r.ld_grad_x = adapter_rows(A, 9, r, r.K, "grad_x");
    float* const ga = A.words<float>(10, r.adapters * r.R * r.K, "grad_a");
    float* const gb = A.words<float>(11, r.adapters * r.R * r.N, "grad_b");
    return invoke(A, fn, &r, A.p(0), A.p(1), A.p(2), t, A.p(7), A.p(8), A.p(9), ga, gb, A.p(12), A.bytes(12), A.stream());
}
int do_adamw_step(Args& A)
{
    FN(fpq_adamw_step);
    const float* const scale = A.words<const float>(8, 1, "grad_scale");
    return invoke(A, fn, A.p(0), A.l(1), A.real(2), A.real(3), A.real(4), A.real(5), A.real(6), A.l(7), scale, A.stream());
}

// ---- blocks, linear layers, gated projections, norm

constexpr int64_t kBlock = 32;
int64_t padded_to(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A matrix of `rows` x `cols` (negative: any; they receive its own) and of `type` (negative: either), or None where that is allowed: its row stride
int64_t matrix(Args& A, int k, int64_t& rows, int64_t& cols, int& type, const char* name, bool optional = false)
{
    if (A.bad || (optional && A.a[k] == Py_None)) return 0;
    if (A.a[k] == Py_None) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor expected", name);
        A.bad = true;
        return 0;
    }
    int64_t n[2] = {}, s[2] = {};
    A.layout(k, 2, n, s, name);
    const int t = A.type(k, name);
    if (A.bad) return 0;
    if (rows < 0) rows = n[0];
    if (cols < 0) cols = n[1];
    if (type < 0) type = t;
    if (n[0] != rows || n[1] != cols || t != type) {
        PyErr_Format(PyExc_ValueError, "%s: %lld rows of %lld elements and one type expected", name, (long long)rows, (long long)cols);
        A.bad = true;
    }
    return s[0];
}
// Contiguous bytes (codes, scales, masks), or None where that is allowed
uint8_t* bytes_of(Args& A, int k, int64_t n, const char* name, bool optional = false)
{
    if (A.bad || (optional && A.a[k] == Py_None)) return nullptr;
    if (A.a[k] == Py_None || A.method(A.a[k], s_numel) != (size_t)n || A.method(A.a[k], s_element_size) != 1) {
        if (!A.bad) PyErr_Format(PyExc_ValueError, "%s: %lld bytes expected", name, (long long)n);
        A.bad = true;
        return nullptr;
    }
    PyObject* c = PyObject_CallMethodNoArgs(A.a[k], s_is_contiguous);
    if (!c || c != Py_True) {
        if (c) PyErr_Format(PyExc_ValueError, "%s: not contiguous", name);
        A.bad = true;
    }
    Py_XDECREF(c);
    return A.bp(k);
}
int do_block_quantize(Args& A)
{
    FN(fpq_block_quantize);
    int64_t M = -1, K = -1;
    int type = -1;
    const int64_t ld = matrix(A, 0, M, K, type, "x");
    const fpq_format_t f = A.fmt(1);
    const int64_t codes = padded_to(K, kBlock) / (1 + f.ebits + f.mbits <= 4 ? 2 : 1);
    const uint8_t* const mask = bytes_of(A, 2, M * K, "mask", true);
    uint8_t *const to = bytes_of(A, 3, M * codes, "codes"), *const scales = bytes_of(A, 4, M * (padded_to(K, kBlock) / kBlock), "scales");
    return invoke(A, fn, A.p(0), type, M, K, ld, f, mask, to, scales, A.stream());
}
int do_block_dequantize(Args& A)
{
    FN(fpq_block_dequantize);
    int64_t M = -1, K = -1;
    int type = -1;
    const int64_t ld = matrix(A, 3, M, K, type, "out");
    const fpq_format_t f = A.fmt(2);
    const int64_t codes = padded_to(K, kBlock) / (1 + f.ebits + f.mbits <= 4 ? 2 : 1);
    const uint8_t *const from = bytes_of(A, 0, M * codes, "codes"), *const scales = bytes_of(A, 1, M * (padded_to(K, kBlock) / kBlock), "scales");
    return invoke(A, fn, from, scales, M, K, f, A.p(3), type, ld, A.stream());
}
int do_block_linear(Args& A)
{
    FN(fpq_block_linear);
    fpq_linear_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.N = r.K = -1;
    int type = -1;
    r.ld_x = matrix(A, 0, r.M, r.K, type, "x");
    r.ld_y = matrix(A, 4, r.M, r.N, type, "y");
    r.type = type;
    const uint8_t *const codes = bytes_of(A, 1, r.N * (padded_to(r.K, kBlock) / 2), "codes"), *const scales = bytes_of(A, 2, r.N * (padded_to(r.K, kBlock) / kBlock), "scales");
    const float* const bias = A.words<const float>(3, r.N, "bias");
    return invoke(A, fn, &r, A.p(0), codes, scales, bias, A.p(4), A.p(5), A.bytes(5), A.stream());
}
// x of a backward call: a matrix [M, K], or its blocks where the scales (the argument behind it) are given; None where no gradient needs it
int64_t kept_rows(Args& A, int k, int64_t& M, int64_t& K, int& type)
{
    if (A.bad || A.a[k] == Py_None) return 0;
    if (A.a[k + 1] == Py_None) return matrix(A, k, M, K, type, "x");
    bytes_of(A, k, M * padded_to(K, kBlock), "x: codes");
    bytes_of(A, k + 1, M * (padded_to(K, kBlock) / kBlock), "x_scales");
    return 0;
}
int do_linear_backward(Args& A)
{
    FN(fpq_linear_backward);
    fpq_linear_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.N = r.K = -1;
    int type = -1;
    r.ld_grad_y = matrix(A, 3, r.M, r.N, type, "grad_y");
    r.ld_w = matrix(A, 2, r.N, r.K, type, "w");
    r.ld_x = kept_rows(A, 0, r.M, r.K, type);
    r.ld_grad_x = matrix(A, 4, r.M, r.K, type, "grad_x", true);
    r.ld_grad_w = matrix(A, 5, r.N, r.K, type, "grad_w", true);
    r.type = type;
    float* const gb = A.words<float>(6, r.N, "grad_bias");
    return invoke(A, fn, &r, A.p(0), (const uint8_t*)A.bp(1), A.p(2), A.p(3), A.p(4), A.p(5), gb, A.p(7), A.bytes(7), A.stream());
}
// What the forward pass keeps: [M, 2 N] of the type, contiguous, or blocks
void kept_pre(Args& A, int k, int64_t M, int64_t N, int type)
{
    if (A.bad || A.a[k] == Py_None) return;
    if (A.a[k + 1] != Py_None) {
        bytes_of(A, k, M * 2 * padded_to(N, kBlock), "pre: codes");
        bytes_of(A, k + 1, M * 2 * (padded_to(N, kBlock) / kBlock), "pre_scales");
        return;
    }
    int64_t cols = 2 * N;
    const int64_t ld = matrix(A, k, M, cols, type, "pre");
    A.same(M <= 1 || ld == cols, "pre: not contiguous");
}
int do_gated(Args& A)
{
    FN(fpq_gated);
    fpq_gated_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.N = r.K = -1;
    int type = -1;
    r.ld_x = matrix(A, 0, r.M, r.K, type, "x");
    r.ld_h = matrix(A, 4, r.M, r.N, type, "h");
    int64_t rows = 2 * r.N;
    r.ld_w = matrix(A, 1, rows, r.K, type, "w");
    r.type = type;
    r.act = A.i(3);
    const float* const bias = A.words<const float>(2, 2 * r.N, "bias");
    kept_pre(A, 5, r.M, r.N, type);
    return invoke(A, fn, &r, A.p(0), A.p(1), bias, A.p(4), A.p(5), A.bp(6), A.p(7), A.bytes(7), A.stream());
}
int do_gated_backward(Args& A)
{
    FN(fpq_gated_backward);
    fpq_gated_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.N = r.K = -1;
    int type = -1;
    r.ld_grad_h = matrix(A, 6, r.M, r.N, type, "grad_h");
    int64_t rows = 2 * r.N;
    r.ld_w = matrix(A, 2, rows, r.K, type, "w");
    r.ld_x = kept_rows(A, 0, r.M, r.K, type);
    r.ld_grad_x = matrix(A, 7, r.M, r.K, type, "grad_x", true);
    r.ld_grad_w = matrix(A, 8, rows, r.K, type, "grad_w", true);
    r.type = type;
    r.act = A.i(5);
    if (!A.bad && A.a[3] == Py_None) {
        PyErr_SetString(PyExc_TypeError, "pre: a tensor expected");
        A.bad = true;
    }
    kept_pre(A, 3, r.M, r.N, type);
    float* const gb = A.words<float>(9, 2 * r.N, "grad_bias");
    return invoke(A, fn, &r, A.p(0), (const uint8_t*)A.bp(1), A.p(2), A.p(3), (const uint8_t*)A.bp(4), A.p(6), A.p(7), A.p(8), gb, A.p(10), A.bytes(10), A.stream());
}
int do_rms_norm(Args& A)
{
    FN(fpq_rms_norm);
    fpq_norm_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.K = -1;
    int type = -1;
    r.ld_x = matrix(A, 0, r.M, r.K, type, "x");
    r.ld_residual = matrix(A, 1, r.M, r.K, type, "residual", true);
    r.ld_sum = matrix(A, 4, r.M, r.K, type, "sum", true);
    r.ld_y = matrix(A, 5, r.M, r.K, type, "y", true);
    r.type = type;
    r.eps = A.f(3);
    const float* const w = A.words<const float>(2, r.K, "w");
    float* const rstd = A.words<float>(6, r.M, "rstd");
    fpq_format_t f;
    memset(&f, 0, sizeof f);
    uint8_t *codes = nullptr, *scales = nullptr;
    float scale = 0.0f;
    const float* dev = nullptr;
    if (A.a[7] != Py_None) {
        const bool blocks = A.a[11] != Py_None;
        codes = bytes_of(A, 7, r.M * padded_to(r.K, blocks ? kBlock : 16), "codes");
        if (blocks) {
            scales = bytes_of(A, 11, r.M * (padded_to(r.K, kBlock) / kBlock), "code_scales");
        } else {
            f = A.fmt(8);
            scale = A.a[9] == Py_None ? 0.0f : A.f(9);
            dev = A.words<const float>(10, 1, "scale_dev");
        }
    } else if (!A.bad && A.a[11] != Py_None) {
        PyErr_SetString(PyExc_ValueError, "code_scales: no codes");
        A.bad = true;
    }
    return invoke(A, fn, &r, A.p(0), A.p(1), w, A.p(4), A.p(5), rstd, codes, f, scale, dev, scales, A.stream());
}
int do_rms_norm_backward(Args& A)
{
    FN(fpq_rms_norm_backward);
    fpq_norm_args_t r;
    memset(&r, 0, sizeof r);
    r.M = r.K = -1;
    int type = -1;
    r.ld_sum = matrix(A, 0, r.M, r.K, type, "sum");
    r.ld_grad_y = matrix(A, 3, r.M, r.K, type, "grad_y");
    r.ld_grad_sum = matrix(A, 4, r.M, r.K, type, "grad_sum", true);
    r.ld_grad_x = matrix(A, 5, r.M, r.K, type, "grad_x", true);
    r.type = type;
    const float *const w = A.words<const float>(1, r.K, "w"), *const rstd = A.words<const float>(2, r.M, "rstd");
    float* const gw = A.words<float>(6, r.K, "grad_w");
    return invoke(A, fn, &r, A.p(0), w, rstd, A.p(3), A.p(4), A.p(5), gw, A.p(7), A.bytes(7), A.stream());
}

// ---- names, parameters and defaults

enum { kMaxParams = 26 };
struct Entry {
    const char* name;
    int (*run)(Args&);
    const char* params;                          // blank-separated
    int required;                                // the others default to 0 ("acc_mode", "causal") or None
    int count;
    PyObject* names[kMaxParams];
    PyObject* defaults[kMaxParams];
};

#define LAYER_HEAD "x x_is_fp32 fx sx sx_dev packed_w fw sw bias "
#define SPARSE_HEAD "x x_is_fp32 fx sx sx_dev packed_sparse fw sw bias "
Entry g_entries[] = {
    {"fpq_gemm", do_gemm, LAYER_HEAD "y M N K acc_mode workspace", 13},
    {"fpq_gemm_noalloc", do_gemm_noalloc, LAYER_HEAD "y M N K acc_mode", 13},
    {"fpq_conv2d", do_conv2d, LAYER_HEAD "y B Cin H W Cout kh kw stride pad acc_mode workspace", 19},
    {"fpq_gemm_codes_out", do_gemm_codes_out, LAYER_HEAD "fy sy sy_dev yq M N K acc_mode workspace", 16},
    {"fpq_conv2d_codes_out", do_conv2d_codes_out, LAYER_HEAD "fy sy sy_dev yq B Cin H W Cout kh kw stride pad acc_mode workspace", 22},
    {"fpq_gemm_sparse", do_gemm_sparse, SPARSE_HEAD "y M N K workspace", 13},
    {"fpq_conv2d_sparse", do_conv2d_sparse, SPARSE_HEAD "y B Cin H W Cout kh kw stride pad workspace", 19},
    {"fpq_gemm_grouped", do_gemm_grouped, "problems x_is_fp32 fx fw acc_mode workspace", 4},
    {"fpq_absmax", do_absmax, "x maxval absmax_out scale_out workspace", 5},
    {"fpq_quantize", do_quantize, "x f scale scale_dev codes", 5},
    {"fpq_quantize_nhwc", do_quantize_nhwc, "x f scale scale_dev codes", 5},
    {"fpq_int_calibrate", do_int_calibrate, "x bits params_out workspace", 4},
    {"fpq_int_quantize", do_int_quantize, "x bits scale zero_point params_dev codes", 6},
    {"fpq_int_gemm", do_int_gemm, "xcodes sx zx px_dev packed_w wbits sw zw bias y M N K workspace", 14},
    {"fpq_rl_step", do_rl_step, "w sw f alpha a lr reg_weight loss_out grad_out workspace", 10},
    {"fpq_search_format", do_search_format, "x encodings n_bias mse_out result workspace", 6},
    {"fpq_attention", do_attention, "q k v o lse scale causal kv_lens workspace", 6},
    {"fpq_attention_backward", do_attention_backward, "q k v o lse grad_o grad_q grad_k grad_v scale causal kv_lens workspace", 10},
    {"fpq_adapter_apply", do_adapter_apply, "x a b scaling row_start adapter base y t workspace", 9},
    {"fpq_adapter_backward", do_adapter_backward,
     "x a b scaling row_start adapter t grad_y grad_x_base grad_x grad_a grad_b workspace", 12},
    {"fpq_adamw_step", do_adamw_step, "plan pieces lr beta1 beta2 eps weight_decay step grad_scale", 8},
    {"fpq_block_quantize", do_block_quantize, "x f mask codes scales", 5},
    {"fpq_block_dequantize", do_block_dequantize, "codes scales f out", 4},
    {"fpq_block_linear", do_block_linear, "x codes scales bias y workspace", 5},
    {"fpq_linear_backward", do_linear_backward, "x x_scales w grad_y grad_x grad_w grad_bias workspace", 7},
    {"fpq_gated", do_gated, "x w bias act h pre pre_scales workspace", 5},
    {"fpq_gated_backward", do_gated_backward, "x x_scales w pre pre_scales act grad_h grad_x grad_w grad_bias workspace", 10},
    {"fpq_rms_norm", do_rms_norm, "x residual w eps sum y rstd codes f scale scale_dev code_scales", 6},
    {"fpq_rms_norm_backward", do_rms_norm_backward, "sum w rstd grad_y grad_sum grad_x grad_w workspace", 7},
};
constexpr int kEntries = sizeof g_entries / sizeof g_entries[0];

PyObject* call_entry(const Entry& e, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)
{
    PyObject* a[kMaxParams];
    if (nargs > e.count) return PyErr_Format(PyExc_TypeError, "%s() takes %d arguments, %zd given", e.name, e.count, nargs);
    for (int k = 0; k < e.count; ++k) a[k] = k < nargs ? args[k] : nullptr;
    if (kwnames) {
        const Py_ssize_t nk = PyTuple_GET_SIZE(kwnames);
        for (Py_ssize_t q = 0; q < nk; ++q) {
            PyObject* name = PyTuple_GET_ITEM(kwnames, q);
            int k = 0;
            while (k < e.count && name != e.names[k] && PyUnicode_Compare(name, e.names[k]) != 0) ++k;
            if (k == e.count) return PyErr_Format(PyExc_TypeError, "%s() has no argument %R", e.name, name);
            if (a[k]) return PyErr_Format(PyExc_TypeError, "%s() got argument %R twice", e.name, name);
            a[k] = args[nargs + q];
        }
    }
    for (int k = 0; k < e.count; ++k)
        if (!a[k] && !(a[k] = e.defaults[k])) return PyErr_Format(PyExc_TypeError, "%s() misses argument %R", e.name, e.names[k]);
    Args A{a};
    const int st = e.run(A);
    if (st == kBad) return nullptr;
    if (st != FPQ_OK) return PyObject_CallFunction(g_check, "is", st, e.name);
    Py_RETURN_NONE;
}

template <int I>
PyObject* trampoline(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames)
{
    return call_entry(g_entries[I], args, nargs, kwnames);
}

PyObject* setup(PyObject*, PyObject* args)
{
    PyObject *r, *c, *f, *p, *a;
    if (!PyArg_ParseTuple(args, "OOOOO", &r, &c, &f, &p, &a)) return nullptr;
    PyObject** const to[] = {&g_resolve, &g_check, &g_format, &g_problem, &g_array};
    PyObject* const from[] = {r, c, f, p, a};
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(from[i]);
        Py_XSETREF(*to[i], from[i]);
    }
    Py_RETURN_NONE;
}

PyMethodDef g_methods[kEntries + 2];

template <int I>
void fill_methods()
{
    if constexpr (I < kEntries) {
        g_methods[I] = PyMethodDef{g_entries[I].name, (PyCFunction)(void (*)(void))trampoline<I>, METH_FASTCALL | METH_KEYWORDS,
                                   g_entries[I].params};
        fill_methods<I + 1>();
    }
}

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fpqcall", "Native argument marshalling of the libfpq binding.", -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fpqcall(void)
{
    s_type = PyUnicode_InternFromString("_type_");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_numel = PyUnicode_InternFromString("numel");
    s_element_size = PyUnicode_InternFromString("element_size");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    PyObject* zero = PyLong_FromLong(0);
    for (int i = 0; i < kEntries; ++i) {
        Entry& e = g_entries[i];
        e.count = 0;
        const char* p = e.params;
        while (*p) {
            const char* q = strchr(p, ' ');
            const size_t len = q ? (size_t)(q - p) : strlen(p);
            PyObject* name = PyUnicode_FromStringAndSize(p, (Py_ssize_t)len);
            PyUnicode_InternInPlace(&name);
            e.names[e.count] = name;
            e.defaults[e.count] = e.count < e.required ? nullptr : (strncmp(p, "acc_mode", 8) == 0 || strncmp(p, "causal", 6) == 0 ? zero : Py_None);
            ++e.count;
            p += len + (q ? 1 : 0);
        }
    }
    fill_methods<0>();
    g_methods[kEntries] = PyMethodDef{"setup", setup, METH_VARARGS, "setup(resolver, checker, fpq_format_t, fpq_gemm_problem_t, ctypes.Array)"};
    g_methods[kEntries + 1] = PyMethodDef{nullptr, nullptr, 0, nullptr};
    return PyModule_Create(&g_module);
}
