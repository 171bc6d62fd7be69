// The run-time calls of binding.py, marshalled natively: tensors in, the C ABI's status out.
//
// A small layer's kernel takes 3 - 5 us.  Marshalling a call in Python -- an attribute check and a pointer object per
// tensor, the current stream, the conversions of a ctypes call -- took 5.5 us beside it, so a program that launches such
// layers one after another waited for its own host thread: 56x56x64 -> 64 3x3 for one image 10.5 us a call.  Here the checks
// are the same ones on the tensor objects themselves, about 0.4 us a call.
//
// Nothing is kept from one call for the next, and nothing is allocated.  The interpreter lock is released around the library
// call (a launch may wait for the device's queue).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

#include "deepgemm_hip.h"

namespace {

PyObject *g_raw_stream = nullptr;        // torch._C._cuda_getCurrentRawStream
PyObject *g_stream_attr = nullptr;       // "cuda_stream"
PyObject *g_address_attr = nullptr;      // "_address"
PyTypeObject *g_desc_type = nullptr;     // binding.ConvDesc, from use_desc
PyTypeObject *g_cache_type = nullptr;    // binding.CacheDesc, the same

struct Failed {};                        // a Python error is set

// One attribute of `o`, or of what it returns when called without arguments; a new reference.
PyObject *attribute(PyObject *o, const char *name, bool call)
{
    PyObject *v = call ? PyObject_CallMethod(o, name, nullptr) : PyObject_GetAttrString(o, name);
    if (!v) throw Failed();
    return v;
}

bool is_true(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Failed();
    return v != 0;
}

// The same for an object that is no torch.Tensor but answers as one (is_cuda, is_contiguous(), dtype, data_ptr()).
void *stand_in_ptr(PyObject *o, at::ScalarType type, const char *name)
{
    if (!PyObject_HasAttrString(o, "is_cuda")) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Failed();
    }
    const char *wrong = nullptr;
    PyObject *v = attribute(o, "is_cuda", false);
    if (!is_true(v)) wrong = "live in device memory";
    Py_DECREF(v);
    if (!wrong) {
        v = attribute(o, "is_contiguous", true);
        if (!is_true(v)) wrong = "be contiguous";
        Py_DECREF(v);
    }
    if (wrong) {
        PyErr_Format(PyExc_ValueError, "%s must %s", name, wrong);
        throw Failed();
    }
    v = attribute(o, "dtype", false);
    const int same = PyObject_RichCompareBool(v, (PyObject *)torch::getTHPDtype(type), Py_EQ);
    if (same == 0) PyErr_Format(PyExc_ValueError, "%s must have dtype %S, got %S", name, (PyObject *)torch::getTHPDtype(type), v);
    Py_DECREF(v);
    if (same != 1) throw Failed();
    v = attribute(o, "data_ptr", true);
    void *ptr = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (!ptr && PyErr_Occurred()) throw Failed();
    return ptr;
}

// The tensor's address; NULL for None.
void *device_ptr(PyObject *o, at::ScalarType type, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) return stand_in_ptr(o, type, name);
    const at::Tensor &t = THPVariable_Unpack(o);
    const char *wrong = !t.is_cuda() ? "live in device memory" : (!t.is_contiguous() ? "be contiguous" : nullptr);
    if (wrong) {
        PyErr_Format(PyExc_ValueError, "%s must %s", name, wrong);
        throw Failed();
    }
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "%s must have dtype %S, got %S", name, (PyObject *)torch::getTHPDtype(type),
                     (PyObject *)torch::getTHPDtype(t.scalar_type()));
        throw Failed();
    }
    return t.data_ptr();
}

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}

// Bytes of a buffer that device_ptr has checked.
size_t bytes_of(PyObject *o)
{
    if (o == Py_None) return 0;
    if (THPVariable_Check(o)) return (size_t)THPVariable_Unpack(o).numel();
    PyObject *v = attribute(o, "numel", true);
    const size_t n = PyLong_AsSize_t(v);
    Py_DECREF(v);
    if (n == (size_t)-1 && PyErr_Occurred()) throw Failed();
    return n;
}

double real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Failed();
    return v;
}

// hipStream_t of a torch stream; None: torch's current stream on the current device.
void *stream_of(PyObject *o)
{
    PyObject *value;
    if (o != Py_None) {
        value = PyObject_GetAttr(o, g_stream_attr);
    } else {
        PyObject *device = PyLong_FromLong(c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index());
        if (!device) throw Failed();
        value = PyObject_CallOneArg(g_raw_stream, device);
        Py_DECREF(device);
    }
    if (!value) throw Failed();
    void *s = PyLong_AsVoidPtr(value);
    Py_DECREF(value);
    if (!s && PyErr_Occurred()) throw Failed();
    return s;
}

// A binding.ConvDesc or CacheDesc as C has it (a ctypes structure lends its memory as a buffer).
template <class Desc>
Desc structure(PyObject *o, PyTypeObject *type, const char *name)
{
    if (!type || !PyObject_TypeCheck(o, type)) {
        PyErr_Format(PyExc_TypeError, "desc must be a %s", name);
        throw Failed();
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Failed();
    Desc d;
    const bool fits = view.len >= (Py_ssize_t)sizeof(d);
    if (fits) memcpy(&d, view.buf, sizeof(d));
    PyBuffer_Release(&view);
    if (!fits) {
        PyErr_Format(PyExc_TypeError, "desc must be a %s", name);
        throw Failed();
    }
    return d;
}
dg_conv_desc geometry(PyObject *o) { return structure<dg_conv_desc>(o, g_desc_type, "ConvDesc"); }
dg_cache_desc cache_geometry(PyObject *o) { return structure<dg_cache_desc>(o, g_cache_type, "CacheDesc"); }

// The table's address: a number, or a binding.Lut's, or the handle of another object that owns a table (a number or a ctypes
// pointer, whose value is None where it is NULL).
const dg_lut *table(PyObject *o)
{
    PyObject *address = nullptr;
    if (PyLong_Check(o)) {
        Py_INCREF(o);
        address = o;
    } else if (PyObject *own = PyObject_GetAttr(o, g_address_attr)) {
        address = own;
    } else {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw Failed();
        PyErr_Clear();
        PyObject *handle = PyObject_GetAttrString(o, "handle");
        if (!handle) {
            PyErr_Format(PyExc_TypeError, "lut must be a table, got %.100s", Py_TYPE(o)->tp_name);
            throw Failed();
        }
        if (PyLong_Check(handle) || handle == Py_None) {
            address = handle;
        } else {
            address = PyObject_GetAttrString(handle, "value");
            Py_DECREF(handle);
            if (!address) throw Failed();
        }
    }
    const size_t value = address == Py_None ? 0 : PyLong_AsSize_t(address);
    Py_DECREF(address);
    if (value == (size_t)-1 && PyErr_Occurred()) throw Failed();
    return (const dg_lut *)value;
}

// Where the result goes: int32, or float32 with a scale or a binary32 table.
struct Output {
    int32_t *i = nullptr;
    float *f = nullptr;
    const float *scale = nullptr;
    Output(PyObject *out, PyObject *scale_o, PyObject *is_f32)
    {
        if (scale_o != Py_None || is_true(is_f32))
            f = (float *)device_ptr(out, at::kFloat, "out");
        else
            i = (int32_t *)device_ptr(out, at::kInt, "out");
        scale = (const float *)device_ptr(scale_o, at::kFloat, "scale");
    }
};

template <class Call>
PyObject *guarded(Py_ssize_t given, Py_ssize_t wanted, Call call)
{
    if (given != wanted) return PyErr_Format(PyExc_TypeError, "%zd arguments, %zd needed", given, wanted);
    try {
        return PyLong_FromLong((long)call());
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The interpreter lock is away while one of these lives.
struct Unlocked {
    PyThreadState *const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// EXPR: the library's call on values that are C's already, nothing of Python's.
#define RUN(EXPR)            \
    const Unlocked unlocked; \
    return EXPR

// (lut, is_f32, Wp, Xp, desc, out, scale, variant, stream)
PyObject *conv2d_lut(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[2], at::kByte, "Wp"), *x = device_ptr(a[3], at::kByte, "Xp");
        const dg_conv_desc d = geometry(a[4]);
        const Output o(a[5], a[6], a[1]);
        const dg_kernel variant = (dg_kernel)integer(a[7]);
        void *s = stream_of(a[8]);
        RUN(dg_conv2d_lut(lut, w, x, &d, o.i, o.scale, o.f, variant, s));
    });
}

// (lut, is_f32, Wp, Xc, desc, work, out, scale, variant, stream)
PyObject *conv2d_lut_codes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[2], at::kByte, "Wp");
        const uint8_t *x = (const uint8_t *)device_ptr(a[3], at::kByte, "Xc");
        const dg_conv_desc d = geometry(a[4]);
        void *work = device_ptr(a[5], at::kByte, "work");
        const Output o(a[6], a[7], a[1]);
        const dg_kernel variant = (dg_kernel)integer(a[8]);
        void *s = stream_of(a[9]);
        const size_t bytes = bytes_of(a[5]);
        RUN(dg_conv2d_lut_codes(lut, w, x, &d, work, bytes, o.i, o.scale, o.f, variant, s));
    });
}

// (lut, is_f32, Wp, Xc, desc, out, scale, variant, stream)
PyObject *conv2d_lut_codes_static(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 9, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[2], at::kByte, "Wp");
        const uint8_t *x = (const uint8_t *)device_ptr(a[3], at::kByte, "Xc");
        const dg_conv_desc d = geometry(a[4]);
        const Output o(a[5], a[6], a[1]);
        const dg_kernel variant = (dg_kernel)integer(a[7]);
        void *s = stream_of(a[8]);
        RUN(dg_conv2d_lut_codes_static(lut, w, x, &d, o.i, o.scale, o.f, variant, s));
    });
}

// (lut, Wp, Xp, desc, scale, q_scale, q_zero, lo, out, variant, stream)
PyObject *conv2d_lut_requant(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[1], at::kByte, "Wp"), *x = device_ptr(a[2], at::kByte, "Xp");
        const dg_conv_desc d = geometry(a[3]);
        const float *scale = (const float *)device_ptr(a[4], at::kFloat, "scale");
        const float qs = (float)real(a[5]), qz = (float)real(a[6]);
        const int32_t lo = (int32_t)integer(a[7]);
        void *out = device_ptr(a[8], at::kByte, "packed");
        const dg_kernel variant = (dg_kernel)integer(a[9]);
        void *s = stream_of(a[10]);
        const size_t bytes = bytes_of(a[8]);
        RUN(dg_conv2d_lut_requant(lut, w, x, &d, scale, qs, qz, lo, out, bytes, variant, s));
    });
}

// (lut, is_f32, Wp, Ap, M, N, K, out, stride_m, stride_n, scale, variant, stream)
PyObject *gemm_lut(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[2], at::kByte, "Wp"), *x = device_ptr(a[3], at::kByte, "Ap");
        const int64_t M = integer(a[4]), N = integer(a[5]), K = integer(a[6]), sm = integer(a[8]), sn = integer(a[9]);
        const Output o(a[7], a[10], a[1]);
        const dg_kernel variant = (dg_kernel)integer(a[11]);
        void *s = stream_of(a[12]);
        RUN(dg_gemm_lut(lut, w, x, M, N, K, o.i, sm, sn, o.scale, o.f, variant, s));
    });
}

// (lut, is_f32, Wp, Ac, M, N, K, work, out, stride_m, stride_n, scale, variant, stream)
PyObject *gemm_lut_codes(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 14, [&] {
        const dg_lut *lut = table(a[0]);
        const void *w = device_ptr(a[2], at::kByte, "Wp");
        const uint8_t *x = (const uint8_t *)device_ptr(a[3], at::kByte, "Ac");
        const int64_t M = integer(a[4]), N = integer(a[5]), K = integer(a[6]), sm = integer(a[9]), sn = integer(a[10]);
        void *work = device_ptr(a[7], at::kByte, "work");
        const Output o(a[8], a[11], a[1]);
        const dg_kernel variant = (dg_kernel)integer(a[12]);
        void *s = stream_of(a[13]);
        const size_t bytes = bytes_of(a[7]);
        RUN(dg_gemm_lut_codes(lut, w, x, M, N, K, work, bytes, o.i, sm, sn, o.scale, o.f, variant, s));
    });
}

// (codes, rows, K, bits, out, stream)
PyObject *pack_codes_bits(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const uint8_t *codes = (const uint8_t *)device_ptr(a[0], at::kByte, "codes");
        const int64_t rows = integer(a[1]), K = integer(a[2]);
        const int32_t bits = (int32_t)integer(a[3]);
        void *out = device_ptr(a[4], at::kByte, "packed");
        void *s = stream_of(a[5]);
        const size_t bytes = bytes_of(a[4]);
        RUN(dg_pack_codes_bits(codes, rows, K, bits, out, bytes, s));
    });
}

// (codes, rows, K, out, stream): weights, activations
template <dg_status (*FN)(const uint8_t *, int64_t, int64_t, void *, size_t, void *)>
PyObject *pack(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const uint8_t *codes = (const uint8_t *)device_ptr(a[0], at::kByte, "codes");
        const int64_t rows = integer(a[1]), K = integer(a[2]);
        void *out = device_ptr(a[3], at::kByte, "packed");
        void *s = stream_of(a[4]);
        const size_t bytes = bytes_of(a[3]);
        RUN(FN(codes, rows, K, out, bytes, s));
    });
}

// (x, N, K, scale, zero_point, lo, out, stream)
PyObject *quantize_pack_activations(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const float *x = (const float *)device_ptr(a[0], at::kFloat, "x");
        const int64_t N = integer(a[1]), K = integer(a[2]);
        const float scale = (float)real(a[3]), zero = (float)real(a[4]);
        const int32_t lo = (int32_t)integer(a[5]);
        void *out = device_ptr(a[6], at::kByte, "packed");
        void *s = stream_of(a[7]);
        const size_t bytes = bytes_of(a[6]);
        RUN(dg_quantize_pack_activations(x, N, K, scale, zero, lo, out, bytes, s));
    });
}

// (acc, rows, C, scale, out, stream)
PyObject *dequantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const int32_t *acc = (const int32_t *)device_ptr(a[0], at::kInt, "acc");
        const int64_t rows = integer(a[1]), C = integer(a[2]);
        const float *scale = (const float *)device_ptr(a[3], at::kFloat, "scale");
        float *out = (float *)device_ptr(a[4], at::kFloat, "out");
        void *s = stream_of(a[5]);
        RUN(dg_dequantize(acc, rows, C, scale, out, s));
    });
}

// ---- a quantised decoder layer: tensors with strides and of several types

// A tensor on the device of `dims` axes, the innermost contiguous.
const at::Tensor &strided(PyObject *o, int dims, const char *name)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Failed();
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must live in device memory", name);
        throw Failed();
    }
    if (t.dim() != dims) {
        PyErr_Format(PyExc_ValueError, "%s must have %d dimensions, got %d", name, dims, (int)t.dim());
        throw Failed();
    }
    if (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous along its last dimension", name);
        throw Failed();
    }
    return t;
}

// Elements from one index of axis `i` to the next; where there is one index at most, what it would be in a contiguous tensor.
int64_t step(const at::Tensor &t, int i)
{
    if (t.size(i) > 1) return t.stride(i);
    int64_t s = 1;
    for (int64_t k = i + 1; k < t.dim(); ++k) s *= t.size(k);
    return s;
}

dg_dtype element_type(const at::Tensor &t, const char *name)
{
    switch (t.scalar_type()) {
    case at::kFloat: return DG_F32;
    case at::kHalf: return DG_F16;
    case at::kBFloat16: return DG_BF16;
    default:
        PyErr_Format(PyExc_ValueError, "%s must have dtype float32, float16 or bfloat16, got %S", name, (PyObject *)torch::getTHPDtype(t.scalar_type()));
        throw Failed();
    }
}

void expect(bool ok, const char *what)
{
    if (ok) return;
    PyErr_SetString(PyExc_ValueError, what);
    throw Failed();
}

const at::Tensor &of_type(const at::Tensor &t, at::ScalarType type, const char *name)
{
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "%s must have dtype %S, got %S", name, (PyObject *)torch::getTHPDtype(type),
                     (PyObject *)torch::getTHPDtype(t.scalar_type()));
        throw Failed();
    }
    return t;
}

// A contiguous vector of `count` elements at least, or NULL for None where that is allowed.
template <class T>
T *vector(PyObject *o, at::ScalarType type, int64_t count, const char *name, bool optional = false)
{
    if (optional && o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw Failed();
    }
    T *p = (T *)device_ptr(o, type, name);
    const int64_t have = THPVariable_Unpack(o).numel();
    if (have < count) {
        PyErr_Format(PyExc_ValueError, "%s must have %lld elements, got %lld", name, (long long)count, (long long)have);
        throw Failed();
    }
    return p;
}

// (x, codes, scale, stream)
PyObject *quantize_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 4, [&] {
        const at::Tensor &x = strided(a[0], 2, "x"), &codes = of_type(strided(a[1], 2, "codes"), at::kChar, "codes");
        const dg_dtype type = element_type(x, "x");
        expect(codes.sizes() == x.sizes(), "codes must have x's shape");
        float *scale = vector<float>(a[2], at::kFloat, x.size(0), "scale");
        void *s = stream_of(a[3]);
        const void *px = x.data_ptr();
        int8_t *pc = (int8_t *)codes.data_ptr();
        const int64_t N = x.size(0), K = x.size(1), sx = step(x, 0), sc = step(codes, 0);
        RUN(dg_quantize_tokens(px, type, N, K, sx, pc, sc, scale, s));
    });
}

// (W, A, scale_m, scale_n, bias, out, stream)
PyObject *gemm_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &W = of_type(strided(a[0], 2, "W"), at::kChar, "W"), &A = of_type(strided(a[1], 2, "A"), at::kChar, "A");
        const at::Tensor &out = strided(a[5], 2, "out");
        const int64_t M = W.size(0), K = W.size(1), N = A.size(0);
        expect(A.size(1) == K, "A and W must have the same number of columns");
        expect(out.size(0) == N && out.size(1) == M, "out must be [tokens][channels]");
        const float *sm = vector<float>(a[2], at::kFloat, M, "scale_m"), *sn = vector<float>(a[3], at::kFloat, N, "scale_n");
        const float *bias = vector<float>(a[4], at::kFloat, M, "bias", true);
        const dg_dtype type = element_type(out, "out");
        void *s = stream_of(a[6]), *po = out.data_ptr();
        const int8_t *pw = (const int8_t *)W.data_ptr(), *pa = (const int8_t *)A.data_ptr();
        const int64_t sw = step(W, 0), sa = step(A, 0), so = step(out, 0);
        RUN(dg_gemm_i8(pw, sw, pa, sa, M, N, K, sm, sn, bias, po, type, so, s));
    });
}

// (W, x, scale_m, bias, work, out, stream)
PyObject *linear_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const at::Tensor &W = of_type(strided(a[0], 2, "W"), at::kChar, "W"), &x = strided(a[1], 2, "x"), &out = strided(a[5], 2, "out");
        const int64_t M = W.size(0), K = W.size(1), N = x.size(0);
        expect(x.size(1) == K, "x and W must have the same number of columns");
        expect(out.size(0) == N && out.size(1) == M, "out must be [tokens][channels]");
        const float *sm = vector<float>(a[2], at::kFloat, M, "scale_m"), *bias = vector<float>(a[3], at::kFloat, M, "bias", true);
        void *work = device_ptr(a[4], at::kByte, "work");
        const size_t bytes = bytes_of(a[4]);
        const dg_dtype xt = element_type(x, "x"), type = element_type(out, "out");
        void *s = stream_of(a[6]), *po = out.data_ptr();
        const void *px = x.data_ptr();
        const int8_t *pw = (const int8_t *)W.data_ptr();
        const int64_t sw = step(W, 0), sx = step(x, 0), so = step(out, 0);
        RUN(dg_linear_i8(pw, sw, px, xt, sx, M, N, K, sm, bias, work, bytes, po, type, so, s));
    });
}

// (desc, cache, k, v, slots, stream)
PyObject *cache_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const dg_cache_desc d = cache_geometry(a[0]);
        void *cache = device_ptr(a[1], at::kByte, "cache");
        const size_t bytes = bytes_of(a[1]);
        const at::Tensor &k = strided(a[2], 3, "k"), &v = strided(a[3], 3, "v");
        const dg_dtype type = element_type(k, "k");
        expect(element_type(v, "v") == type && v.sizes() == k.sizes(), "k and v must have one shape and dtype");
        expect(k.size(1) == d.heads && k.size(2) == d.dim, "k and v must be [tokens][heads][dim]");
        const int64_t T = k.size(0), kt = step(k, 0), kh = step(k, 1), vt = step(v, 0), vh = step(v, 1);
        const int32_t *slots = vector<int32_t>(a[4], at::kInt, T, "slots");
        void *s = stream_of(a[5]);
        const void *pk = k.data_ptr(), *pv = v.data_ptr();
        RUN(dg_cache_write(&d, cache, bytes, pk, pv, type, T, kt, kh, vt, vh, slots, s));
    });
}

// (desc, cache, slots, k_out, v_out, stream)
PyObject *cache_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const dg_cache_desc d = cache_geometry(a[0]);
        void *cache = device_ptr(a[1], at::kByte, "cache");
        const size_t bytes = bytes_of(a[1]);
        const int32_t *slots = vector<int32_t>(a[2], at::kInt, 0, "slots");
        const int64_t T = THPVariable_Unpack(a[2]).numel();
        void *out[2] = {nullptr, nullptr};
        dg_dtype type = DG_F32;
        bool first = true;
        for (int i = 0; i < 2; ++i) {
            if (a[3 + i] == Py_None) continue;
            const at::Tensor &t = strided(a[3 + i], 3, i ? "v_out" : "k_out");
            const dg_dtype its = element_type(t, i ? "v_out" : "k_out");
            expect(first || its == type, "k_out and v_out must have one dtype");
            expect(t.is_contiguous() && t.size(0) == T && t.size(1) == d.heads && t.size(2) == d.dim,
                   "k_out and v_out must be contiguous [slots][heads][dim]");
            type = its;
            first = false;
            out[i] = t.data_ptr();
        }
        void *s = stream_of(a[5]);
        RUN(dg_cache_read(&d, cache, bytes, slots, T, out[0], out[1], type, s));
    });
}

// (desc, cache, q, q_start, ctx_len, table, max_q, max_ctx, scale, causal, out, work, stream)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 13, [&] {
        const dg_cache_desc d = cache_geometry(a[0]);
        void *cache = device_ptr(a[1], at::kByte, "cache");
        const size_t bytes = bytes_of(a[1]);
        const at::Tensor &q = strided(a[2], 3, "q"), &out = strided(a[10], 3, "out"), &table = of_type(strided(a[5], 2, "table"), at::kInt, "table");
        const dg_dtype type = element_type(q, "q");
        expect(element_type(out, "out") == type && out.sizes() == q.sizes(), "out must have q's shape and dtype");
        expect(q.size(2) == d.dim, "q must be [tokens][query heads][dim]");
        expect(table.is_contiguous(), "table must be contiguous");
        const int64_t T = q.size(0), Hq = q.size(1), B = table.size(0), width = table.size(1);
        const int32_t *start = vector<int32_t>(a[3], at::kInt, B + 1, "q_start"), *ctx = vector<int32_t>(a[4], at::kInt, B, "ctx_len");
        const int64_t max_q = integer(a[6]), max_ctx = integer(a[7]);
        const float scale = (float)real(a[8]);
        const int32_t causal = is_true(a[9]);
        void *work = device_ptr(a[11], at::kByte, "work");
        const size_t work_bytes = bytes_of(a[11]);
        void *s = stream_of(a[12]), *po = out.data_ptr();
        const void *pq = q.data_ptr();
        const int32_t *pt = (const int32_t *)table.data_ptr();
        const int64_t qt = step(q, 0), qh = step(q, 1), ot = step(out, 0), oh = step(out, 1);
        RUN(dg_paged_attention(&d, cache, bytes, pq, type, T, Hq, qt, qh, start, ctx, pt, B, width, max_q, max_ctx, scale, causal, po, ot, oh, work,
                               work_bytes, s));
    });
}

// (ConvDesc, CacheDesc): binding's types, whose instances alone are taken for a geometry
PyObject *use_desc(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 2, [&] {
        if (!PyType_Check(a[0]) || !PyType_Check(a[1])) {
            PyErr_SetString(PyExc_TypeError, "a type is needed");
            throw Failed();
        }
        Py_INCREF(a[0]);
        Py_XDECREF((PyObject *)g_desc_type);
        g_desc_type = (PyTypeObject *)a[0];
        Py_INCREF(a[1]);
        Py_XDECREF((PyObject *)g_cache_type);
        g_cache_type = (PyTypeObject *)a[1];
        return 0;
    });
}

#define METHOD(NAME, FN) {NAME, (PyCFunction)(void (*)(void))(FN), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD("conv2d_lut", conv2d_lut), METHOD("conv2d_lut_codes", conv2d_lut_codes),
    METHOD("conv2d_lut_codes_static", conv2d_lut_codes_static), METHOD("conv2d_lut_requant", conv2d_lut_requant),
    METHOD("gemm_lut", gemm_lut), METHOD("gemm_lut_codes", gemm_lut_codes), METHOD("pack_codes_bits", pack_codes_bits),
    METHOD("pack_weights", pack<dg_pack_weights>), METHOD("pack_activations", pack<dg_pack_activations>),
    METHOD("quantize_pack_activations", quantize_pack_activations), METHOD("dequantize", dequantize),
    METHOD("quantize_tokens", quantize_tokens), METHOD("gemm_i8", gemm_i8), METHOD("linear_i8", linear_i8),
    METHOD("cache_write", cache_write), METHOD("cache_read", cache_read), METHOD("paged_attention", paged_attention),
    METHOD("use_desc", use_desc),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", "Tensors in, the C ABI's status out.", -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

}   // namespace

PyMODINIT_FUNC PyInit__native()
{
    PyObject *torch_c = PyImport_ImportModule("torch._C");
    if (!torch_c) return nullptr;
    g_raw_stream = PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream");
    Py_DECREF(torch_c);
    g_stream_attr = PyUnicode_InternFromString("cuda_stream");
    g_address_attr = PyUnicode_InternFromString("_address");
    if (!g_raw_stream || !g_stream_attr || !g_address_attr) return nullptr;
    return PyModule_Create(&module_def);
}
