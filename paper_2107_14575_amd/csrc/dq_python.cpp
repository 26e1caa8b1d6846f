// The Python side of the per-iteration entry points: takes the tensors' addresses, strides and row counts and calls the C
// functions of dq.h, without the GIL.  The functions are those of the library that binding.py has opened, which hands their addresses over
// (bind): the module itself needs no libdq.so, so it cannot come by another one on the loader's search path or of another copy of the
// package, whose plans have another form.  Arguments are converted as ctypes
// converts them: plain numbers here, and whatever else it takes (numpy's and torch's numbers, instances of the C types, objects with
// _as_parameter_) or refuses (ctypes.ArgumentError) by ctypes itself.  Returns the status; binding.py has the names, defaults and checks.
//
// A small call is its launch (2.6 us of HIP) and what leads there.  Through ctypes, with the attributes read in Python:
// quantize_pack 5.5 us, norm 4.8, select_bits 2.0; here 4.6, 4.1, 0.4.  An iteration of 4096 values, M = 8, 33.8 -> 28.9 us, of 2^20, M = 4,
// 35.9 -> 31.9.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include <new>
#include <vector>

#include "dq.h"

namespace {

#define DQ_FUNCTIONS(X) \
    X(dq_norm) X(dq_norm_linf) X(dq_quantize_pack) X(dq_quantize_pack_v) X(dq_norm_quantize_pack) X(dq_norm_bracket) \
    X(dq_norm_quantize_pack_bracketed) X(dq_norm_quantize_pack_bracketed_v) X(dq_unpack_dequant_reduce) X(dq_unpack_dequant_reduce_v) \
    X(dq_unpack_dequant_reduce_update) X(dq_unpack_dequant_reduce_update_v) X(dq_sign_pack) X(dq_sign_reduce) X(dq_sign_majority) \
    X(dq_select_bits) X(dq_select_bits_linf) X(dq_packed_bytes) X(dq_token_logprob) X(dq_token_logprob_backward) X(dq_policy_loss) \
    X(dq_preference_loss) X(dq_token_logprob_workspace_bytes) X(dq_policy_loss_workspace_bytes) X(dq_preference_loss_workspace_bytes) \
    X(dq_grad_norm) X(dq_clip_grads) X(dq_clip_gather) X(dq_clip_norms) X(dq_clip_workspace_bytes) X(dq_clip_norms_workspace_bytes) \
    X(dq_plan_num_segments)

enum { INT32, UINT32, INT64, UINT64, ADDRESS, FLOAT32, FLOAT64, N_KINDS };

// Of one module object: copies of the package that share this file are bound each to their own library.
struct state {
#define X(fn) decltype(&::fn) fn;
    DQ_FUNCTIONS(X)
#undef X
    bool bound;
    PyObject* convert[N_KINDS]; // ctypes functions of one argument, which they return
    PyObject *data_ptr, *stride, *size, *shape, *zero;
    PyObject *dtype, *numel, *element_size, *get_device, *is_contiguous;
    PyObject* types[4]; // torch's float32, float16, bfloat16 (as dq_dtype counts them) and int64; null until torch is there (set_types)
};
state* state_of(PyObject* module) { return static_cast<state*>(PyModule_GetState(module)); }

// One call's arguments, taken one after the other; `ok` goes false with a Python exception set.
struct taker {
    const state* lib;
    PyObject* const* args;
    Py_ssize_t at = 0;
    bool ok = true;

    taker(PyObject* module, PyObject* const* a, Py_ssize_t have, Py_ssize_t want) : lib(state_of(module)), args(a)
    {
        if (!lib->bound) {
            PyErr_SetString(PyExc_RuntimeError, "no library bound");
            ok = false;
        } else if (have != want) {
            PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, have);
            ok = false;
        }
    }
    PyObject* converted(int kind, PyObject* o) // as ctypes passes it; a new reference
    {
        PyObject* value = PyObject_CallOneArg(lib->convert[kind], o);
        if (!value) ok = false;
        return value;
    }
    uint64_t bits_of(int kind, PyObject* o)
    {
        if (PyLong_Check(o)) return PyLong_AsUnsignedLongLongMask(o); // no error: an int
        PyObject* value = converted(kind, o);
        if (!value) return 0;
        const uint64_t v = PyLong_AsUnsignedLongLongMask(value);
        Py_DECREF(value);
        return v;
    }
    int64_t int_of(PyObject* o) // int(o); takes the reference
    {
        if (o && !PyLong_Check(o)) {
            PyObject* value = PyNumber_Long(o);
            Py_DECREF(o);
            o = value;
        }
        if (!o) {
            ok = false;
            return 0;
        }
        const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
        Py_DECREF(o);
        return static_cast<int64_t>(v);
    }
    uint64_t whole(int kind) { return ok ? bits_of(kind, args[at++]) : 0; }
    int as_int() { return static_cast<int>(whole(INT32)); }
    uint32_t as_u32() { return static_cast<uint32_t>(whole(UINT32)); }
    int64_t as_i64() { return static_cast<int64_t>(whole(INT64)); }
    uint64_t as_u64() { return whole(UINT64); }
    void* address() { return reinterpret_cast<void*>(whole(ADDRESS)); } // a handle or stream
    double real(int kind)
    {
        if (!ok) return 0.0;
        PyObject* o = args[at++];
        if (PyFloat_Check(o)) return PyFloat_AS_DOUBLE(o);
        PyObject* value = converted(kind, o);
        if (!value) return 0.0;
        const double v = PyFloat_AsDouble(value);
        Py_DECREF(value);
        return v;
    }
    float as_float() { return static_cast<float>(real(FLOAT32)); }
    double as_double() { return real(FLOAT64); }
    PyObject* object() { return ok ? args[at++] : nullptr; }
    template <typename T>
    T* data_of(PyObject* t) // NULL for None
    {
        if (!ok || t == Py_None) return nullptr;
        PyObject* at_address = PyObject_CallMethodNoArgs(t, lib->data_ptr);
        if (!at_address) {
            ok = false;
            return nullptr;
        }
        const uint64_t v = bits_of(ADDRESS, at_address);
        Py_DECREF(at_address);
        return reinterpret_cast<T*>(v);
    }
    template <typename T>
    T* data()
    {
        PyObject* t = object();
        if (ok && t == Py_None) { // as None.data_ptr()
            PyErr_SetString(PyExc_AttributeError, "'NoneType' object has no attribute 'data_ptr'");
            ok = false;
        }
        return data_of<T>(t);
    }
    template <typename T>
    T* data_or_null()
    {
        return data_of<T>(object());
    }
    int64_t stride0(PyObject* t) { return ok ? int_of(PyObject_CallMethodOneArg(t, lib->stride, lib->zero)) : 0; }
    int rows(PyObject* t)
    {
        if (!ok) return 0;
        if (PyObject* size = PyObject_CallMethodOneArg(t, lib->size, lib->zero)) return static_cast<int>(int_of(size));
        if (!PyErr_ExceptionMatches(PyExc_Exception)) {
            ok = false;
            return 0;
        }
        PyErr_Clear(); // no size(0), as a tensor has: shape[0]
        PyObject* shape = PyObject_GetAttr(t, lib->shape);
        PyObject* first = shape ? PyObject_GetItem(shape, lib->zero) : nullptr;
        Py_XDECREF(shape);
        return static_cast<int>(int_of(first));
    }
};

template <typename F>
PyObject* status_of(const taker& a, F&& call)
{
    if (!a.ok) return nullptr;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = call();
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

template <typename T>
struct matrix { // a tensor of one row per worker
    T* data;
    int64_t stride;
    int rows;
};
template <typename T>
matrix<T> take_matrix(taker& a)
{
    PyObject* t = a.object();
    matrix<T> m = {};
    if (!a.ok) return m;
    m.rows = a.rows(t);
    m.stride = a.stride0(t);
    m.data = a.data_of<T>(t);
    return m;
}

using args_t = PyObject* const*;

// (plan, grads, norms, workspace, linf, stream)
PyObject* py_norm(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 6);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    float* norms = a.data<float>();
    void* workspace = a.data<void>();
    const int linf = a.as_int();
    void* stream = a.address();
    return status_of(a, [&] {
        return linf ? a.lib->dq_norm_linf(plan, grads.data, grads.stride, grads.rows, norms, workspace, stream)
                    : a.lib->dq_norm(plan, grads.data, grads.stride, grads.rows, norms, workspace, stream);
    });
}

// (plan, grads, norms, b, seed, step, worker_base, packed, stream)
PyObject* py_quantize_pack(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 9);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    const float* norms = a.data<const float>();
    const int b = a.as_int();
    const uint64_t seed = a.as_u64();
    const uint32_t step = a.as_u32(), worker_base = a.as_u32();
    PyObject* out = a.object();
    uint8_t* packed = a.data_of<uint8_t>(out);
    const int64_t stride = a.stride0(out);
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_quantize_pack(plan, grads.data, grads.stride, grads.rows, norms, b, seed, step, worker_base, packed, stride, stream);
    });
}

// (plan, widths, grads, norms, seed, step, worker_base, packed, stream)
PyObject* py_quantize_pack_v(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 9);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto* widths = static_cast<const dq_widths_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    const float* norms = a.data<const float>();
    const uint64_t seed = a.as_u64();
    const uint32_t step = a.as_u32(), worker_base = a.as_u32();
    PyObject* out = a.object();
    uint8_t* packed = a.data_of<uint8_t>(out);
    const int64_t stride = a.stride0(out);
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_quantize_pack_v(plan, widths, grads.data, grads.stride, grads.rows, norms, seed, step, worker_base, packed, stride,
                                  stream);
    });
}

// (plan, grads, b, seed, step, worker_base, norms, packed, linf, stream)
PyObject* py_norm_quantize_pack(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 10);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    const int b = a.as_int();
    const uint64_t seed = a.as_u64();
    const uint32_t step = a.as_u32(), worker_base = a.as_u32();
    float* norms = a.data<float>();
    PyObject* out = a.object();
    uint8_t* packed = a.data_of<uint8_t>(out);
    const int64_t stride = a.stride0(out);
    const int linf = a.as_int();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_norm_quantize_pack(plan, grads.data, grads.stride, grads.rows, linf, b, seed, step, worker_base, norms, packed, stride,
                                     stream);
    });
}

// (norms, numel, margin, lo, hi, stream)
PyObject* py_norm_bracket(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 6);
    const float* norms = a.data<const float>();
    const int64_t count = a.as_i64();
    const float margin = a.as_float();
    float *lo = a.data<float>(), *hi = a.data<float>();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_norm_bracket(norms, count, margin, lo, hi, stream); });
}

// (plan, widths or 0, grads, lo, hi, b, seed, step, worker_base, norms, packed, workspace, stats, linf, stream)
PyObject* py_bracketed(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 15);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto* widths = static_cast<const dq_widths_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    const float *lo = a.data<const float>(), *hi = a.data<const float>();
    const int b = a.as_int();
    const uint64_t seed = a.as_u64();
    const uint32_t step = a.as_u32(), worker_base = a.as_u32();
    float* norms = a.data<float>();
    PyObject* out = a.object();
    uint8_t* packed = a.data_of<uint8_t>(out);
    const int64_t stride = a.stride0(out);
    void* workspace = a.data<void>();
    auto* stats = a.data_or_null<int64_t>();
    const int linf = a.as_int();
    void* stream = a.address();
    return status_of(a, [&] {
        return widths ? a.lib->dq_norm_quantize_pack_bracketed_v(plan, widths, grads.data, grads.stride, grads.rows, linf, lo, hi, seed, step,
                                                          worker_base, norms, packed, stride, workspace, stats, stream)
                      : a.lib->dq_norm_quantize_pack_bracketed(plan, grads.data, grads.stride, grads.rows, linf, lo, hi, b, seed, step,
                                                        worker_base, norms, packed, stride, workspace, stats, stream);
    });
}

// (plan, packed, norms, b, out, stream)
PyObject* py_reduce(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 6);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto packed = take_matrix<const uint8_t>(a);
    const float* norms = a.data<const float>();
    const int b = a.as_int();
    float* out = a.data<float>();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_unpack_dequant_reduce(plan, packed.data, packed.stride, packed.rows, norms, b, out, stream); });
}

// (plan, packed, norms, b, eta, x, ghat, stream)
PyObject* py_reduce_update(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 8);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto packed = take_matrix<const uint8_t>(a);
    const float* norms = a.data<const float>();
    const int b = a.as_int();
    const float eta = a.as_float();
    float *x = a.data<float>(), *ghat = a.data_or_null<float>();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_unpack_dequant_reduce_update(plan, packed.data, packed.stride, packed.rows, norms, b, eta, x, ghat, stream);
    });
}

// (plan, widths, packed, norms, out, stream)
PyObject* py_reduce_v(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 6);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto* widths = static_cast<const dq_widths_t*>(a.address());
    const auto packed = take_matrix<const uint8_t>(a);
    const float* norms = a.data<const float>();
    float* out = a.data<float>();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_unpack_dequant_reduce_v(plan, widths, packed.data, packed.stride, packed.rows, norms, out, stream); });
}

// (plan, widths, packed, norms, eta, x, ghat, stream)
PyObject* py_reduce_update_v(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 8);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto* widths = static_cast<const dq_widths_t*>(a.address());
    const auto packed = take_matrix<const uint8_t>(a);
    const float* norms = a.data<const float>();
    const float eta = a.as_float();
    float *x = a.data<float>(), *ghat = a.data_or_null<float>();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_unpack_dequant_reduce_update_v(plan, widths, packed.data, packed.stride, packed.rows, norms, eta, x, ghat, stream);
    });
}

// (plan, grads, packed, stream)
PyObject* py_sign_pack(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 4);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto grads = take_matrix<const float>(a);
    PyObject* out = a.object();
    uint8_t* packed = a.data_of<uint8_t>(out);
    const int64_t stride = a.stride0(out);
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_sign_pack(plan, grads.data, grads.stride, grads.rows, packed, stride, stream); });
}

// (plan, packed, scales, out, majority, stream)
PyObject* py_sign_reduce(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 6);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto packed = take_matrix<const uint8_t>(a);
    const float* scales = a.data_or_null<const float>();
    float* out = a.data<float>();
    const int majority = a.as_int();
    void* stream = a.address();
    return status_of(a, [&] {
        return majority ? a.lib->dq_sign_majority(plan, packed.data, packed.stride, packed.rows, out, stream)
                        : a.lib->dq_sign_reduce(plan, packed.data, packed.stride, packed.rows, scales, out, stream);
    });
}

// (norms: C-contiguous float32 [M][n_seg], t, T, eps_hat_q, alpha, b_min, b_max, linf) -> (status, b, Gbar)
PyObject* py_select_bits(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 8);
    PyObject* array = a.object();
    const int64_t t = a.as_i64(), T = a.as_i64();
    const double eps = a.as_double(), alpha = a.as_double();
    const int b_min = a.as_int(), b_max = a.as_int(), linf = a.as_int();
    if (!a.ok) return nullptr;
    Py_buffer view;
    if (PyObject_GetBuffer(array, &view, PyBUF_C_CONTIGUOUS) != 0) return nullptr;
    if (view.ndim != 2 || view.itemsize != 4 || view.shape[0] > INT32_MAX || view.shape[1] > INT32_MAX) {
        PyBuffer_Release(&view);
        PyErr_SetString(PyExc_ValueError, "norms must be [M][n_seg]");
        return nullptr;
    }
    int b = 0, status;
    double gbar = 0.0;
    const auto* norms = static_cast<const float*>(view.buf);
    const int M = static_cast<int>(view.shape[0]), n_seg = static_cast<int>(view.shape[1]);
    Py_BEGIN_ALLOW_THREADS;
    status = linf ? a.lib->dq_select_bits_linf(norms, M, n_seg, t, T, eps, alpha, b_min, b_max, &b, &gbar)
                  : a.lib->dq_select_bits(norms, M, n_seg, t, T, eps, alpha, b_min, b_max, &b, &gbar);
    Py_END_ALLOW_THREADS;
    PyBuffer_Release(&view);
    return Py_BuildValue("iid", status, b, gbar);
}

// (plan, b) -> bytes
PyObject* py_packed_bytes(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 2);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const int b = a.as_int();
    if (!a.ok) return nullptr;
    return PyLong_FromLongLong(a.lib->dq_packed_bytes(plan, b));
}

// ---- the operators between logits and gradients, and clipping.  Their arguments are checked here, for type, size, layout and GPU, in the order of the
// call: what a kernel is given has the elements that it reads.
enum { KIND_F32 = DQ_F32, KIND_F16 = DQ_F16, KIND_BF16 = DQ_BF16, KIND_INT64 = 3, KINDS = 4 };

struct checker {
    taker& a;
    int64_t device; // the current one

    checker(taker& taken, int64_t current) : a(taken), device(current)
    {
        if (a.ok && !a.lib->types[0]) {
            PyErr_SetString(PyExc_RuntimeError, "no types set");
            a.ok = false;
        }
    }
    void refuse(const char* name, const char* what)
    {
        if (a.ok) PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
        a.ok = false;
    }
    int64_t number(PyObject* t, PyObject* method) { return a.ok ? a.int_of(PyObject_CallMethodNoArgs(t, method)) : 0; }
    bool truth(PyObject* t, PyObject* method)
    {
        if (!a.ok) return false;
        PyObject* r = PyObject_CallMethodNoArgs(t, method);
        const int yes = r ? PyObject_IsTrue(r) : -1;
        Py_XDECREF(r);
        if (yes < 0) a.ok = false;
        return yes > 0;
    }
    int kind(PyObject* t)
    {
        if (!a.ok) return -1;
        PyObject* type = PyObject_GetAttr(t, a.lib->dtype);
        if (!type) {
            a.ok = false;
            return -1;
        }
        int k = 0;
        while (k < KINDS && a.lib->types[k] != type) ++k;
        Py_DECREF(type);
        return k;
    }
    void here(PyObject* t, const char* name)
    {
        if (a.ok && number(t, a.lib->get_device) != device) refuse(name, "not on the current GPU");
    }
    // the next argument: a contiguous tensor of `count` elements of one type, or None where that may be
    template <typename T>
    T* array(const char* name, int want, int64_t count, bool may_be_none = false)
    {
        PyObject* t = a.object();
        if (!a.ok || (t == Py_None && may_be_none)) return nullptr;
        if (kind(t) != want && a.ok) refuse(name, want == KIND_INT64 ? "int64 is wanted" : "float32 is wanted");
        if (a.ok && number(t, a.lib->numel) != count) refuse(name, "has another number of elements");
        if (a.ok && !truth(t, a.lib->is_contiguous)) refuse(name, "not contiguous");
        here(t, name);
        return a.data_of<T>(t);
    }
    void* workspace(int64_t bytes)
    {
        PyObject* t = a.object();
        const int64_t have = number(t, a.lib->numel) * number(t, a.lib->element_size);
        if (a.ok && (bytes < 0 || have < bytes)) refuse("workspace", "too small: see the *_workspace_bytes function");
        if (a.ok && !truth(t, a.lib->is_contiguous)) refuse("workspace", "not contiguous");
        here(t, "workspace");
        return a.data_of<void>(t);
    }
    // [rows][vocab] or [batch][rows][vocab]
    bool logits(const char* name, dq_logits_t& m, bool may_be_none = false)
    {
        m = {};
        PyObject* t = a.object();
        if (!a.ok || (t == Py_None && may_be_none)) return false;
        m.dtype = kind(t);
        if (a.ok && m.dtype > DQ_BF16) refuse(name, "float32, float16 or bfloat16 is wanted");
        int64_t sizes[3] = { 1, 0, 0 }, strides[3] = { 0, 0, 0 };
        Py_ssize_t n = 0;
        for (int what = 0; what < 2 && a.ok; ++what) {
            PyObject* tuple = what ? PyObject_CallMethodNoArgs(t, a.lib->stride) : PyObject_GetAttr(t, a.lib->shape);
            if (!tuple || !PyTuple_Check(tuple)) {
                if (tuple) PyErr_SetString(PyExc_TypeError, "a tensor is wanted");
                a.ok = false;
            } else {
                n = PyTuple_GET_SIZE(tuple);
                if (n != 2 && n != 3) refuse(name, "[rows][vocab] or [batch][rows][vocab] is wanted");
                for (Py_ssize_t k = 0; k < n && a.ok; ++k) {
                    PyObject* v = PyTuple_GET_ITEM(tuple, k);
                    Py_INCREF(v);
                    (what ? strides : sizes)[3 - n + k] = a.int_of(v);
                }
            }
            Py_XDECREF(tuple);
        }
        if (a.ok && sizes[2] > 1 && strides[2] != 1) refuse(name, "the vocabulary has to be the contiguous dimension");
        here(t, name);
        m.batch = sizes[0];
        m.rows = sizes[1];
        m.vocab = sizes[2];
        m.batch_stride = strides[0];
        m.row_stride = strides[1];
        m.data_dev = a.data_of<void>(t);
        return a.ok;
    }
    void same_sizes(const dq_logits_t& m, const dq_logits_t& gradient)
    {
        if (a.ok && (m.dtype != gradient.dtype || m.batch != gradient.batch || m.rows != gradient.rows || m.vocab != gradient.vocab))
            refuse("dlogits", "has another type or another size than the logits");
    }
};

// (logits, tokens, logp, softmax or None, workspace, temperature, device, stream)
PyObject* py_token_logprob(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 8);
    checker c(a, a.ok ? PyLong_AsLongLong(args[6]) : 0);
    dq_logits_t m;
    c.logits("logits", m);
    const int64_t rows = m.batch * m.rows;
    const auto* tokens = c.array<const int64_t>("tokens", KIND_INT64, rows);
    auto* logp = c.array<float>("logp", KIND_F32, rows);
    auto* softmax = c.array<float>("softmax", KIND_F32, 2 * rows, true);
    void* workspace = c.workspace(a.ok ? a.lib->dq_token_logprob_workspace_bytes(rows, m.vocab) : 0);
    const double temperature = a.as_double();
    a.object();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_token_logprob(&m, tokens, temperature, logp, softmax, workspace, stream); });
}

// (logits, tokens, softmax, dlogp, dlogits, temperature, grad_scale, device, stream)
PyObject* py_token_logprob_backward(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 9);
    checker c(a, a.ok ? PyLong_AsLongLong(args[7]) : 0);
    dq_logits_t m, g;
    c.logits("logits", m);
    const int64_t rows = m.batch * m.rows;
    const auto* tokens = c.array<const int64_t>("tokens", KIND_INT64, rows);
    const auto* softmax = c.array<const float>("softmax", KIND_F32, 2 * rows);
    const auto* dlogp = c.array<const float>("dlogp", KIND_F32, rows);
    c.logits("dlogits", g);
    c.same_sizes(m, g);
    const double temperature = a.as_double(), scale = a.as_double();
    a.object();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_token_logprob_backward(&m, tokens, temperature, softmax, dlogp, scale, &g, stream); });
}

// (logits, tokens, old_logp, ref_logp or None, advantages, weights, loss, logp, dlogits or None, workspace, clip_low, clip_high, beta, temperature,
//  grad_scale, device, stream)
PyObject* py_policy_loss(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 17);
    checker c(a, a.ok ? PyLong_AsLongLong(args[15]) : 0);
    dq_logits_t m, g;
    c.logits("logits", m);
    const int64_t rows = m.batch * m.rows;
    const auto* tokens = c.array<const int64_t>("tokens", KIND_INT64, rows);
    const auto* old_logp = c.array<const float>("old_logp", KIND_F32, rows);
    const auto* ref_logp = c.array<const float>("ref_logp", KIND_F32, rows, true);
    const auto* advantages = c.array<const float>("advantages", KIND_F32, rows);
    const auto* weights = c.array<const float>("weights", KIND_F32, rows);
    auto* loss = c.array<float>("loss", KIND_F32, 4);
    auto* logp = c.array<float>("logp", KIND_F32, rows);
    const bool gradient = c.logits("dlogits", g, true);
    if (gradient) c.same_sizes(m, g);
    void* workspace = c.workspace(a.ok ? a.lib->dq_policy_loss_workspace_bytes(rows, m.vocab) : 0);
    const double low = a.as_double(), high = a.as_double(), beta = a.as_double(), temperature = a.as_double(), scale = a.as_double();
    a.object();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_policy_loss(&m, tokens, temperature, old_logp, ref_logp, advantages, weights, low, high, beta, scale, loss, logp, gradient ? &g : nullptr,
                                     workspace, stream);
    });
}

// (logits, tokens, seq_start, pairs, ref_logp or None, loss, seq_logp, dlogits or None, workspace, beta, label_smoothing, average, temperature,
//  grad_scale, device, stream)
PyObject* py_preference_loss(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 16);
    checker c(a, a.ok ? PyLong_AsLongLong(args[14]) : 0);
    const int64_t pairs = a.ok ? PyLong_AsLongLong(args[3]) : 0;
    dq_logits_t m, g;
    c.logits("logits", m);
    const int64_t rows = m.batch * m.rows;
    const auto* tokens = c.array<const int64_t>("tokens", KIND_INT64, rows);
    const auto* seq_start = c.array<const int64_t>("seq_start", KIND_INT64, 2 * pairs + 1);
    a.object();
    const auto* ref_logp = c.array<const float>("ref_logp", KIND_F32, 2 * pairs, true);
    auto* loss = c.array<float>("loss", KIND_F32, 4);
    auto* seq_logp = c.array<float>("seq_logp", KIND_F32, 2 * pairs);
    const bool gradient = c.logits("dlogits", g, true);
    if (gradient) c.same_sizes(m, g);
    void* workspace = c.workspace(a.ok ? a.lib->dq_preference_loss_workspace_bytes(rows, m.vocab, pairs) : 0);
    const double beta = a.as_double(), smoothing = a.as_double();
    const int average = a.as_int();
    const double temperature = a.as_double(), scale = a.as_double();
    a.object();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_preference_loss(&m, tokens, temperature, seq_start, pairs, ref_logp, beta, smoothing, average, scale, loss, seq_logp,
                                         gradient ? &g : nullptr, workspace, stream);
    });
}

// A list of tensors: their addresses, lengths and types.
struct tensor_list {
    std::vector<void*> data;
    std::vector<int64_t> len;
    std::vector<int32_t> type;

    void take(checker& c, const char* name)
    {
        taker& a = c.a;
        PyObject* list = a.object();
        PyObject* sequence = a.ok ? PySequence_Fast(list, "a list of tensors is wanted") : nullptr;
        // a tuple, which holds its tensors: their methods may be any code, and the list could change
        PyObject* items = sequence ? PySequence_Tuple(sequence) : nullptr;
        Py_XDECREF(sequence);
        if (!items) {
            a.ok = false;
            return;
        }
        const Py_ssize_t n = PyTuple_GET_SIZE(items);
        try {
            data.reserve(n);
            len.reserve(n);
            type.reserve(n);
        } catch (const std::bad_alloc&) {
            PyErr_NoMemory();
            a.ok = false;
        }
        if (n > INT32_MAX) c.refuse(name, "too many tensors");
        for (Py_ssize_t i = 0; i < n && a.ok; ++i) {
            PyObject* t = PyTuple_GET_ITEM(items, i);
            const int kind = c.kind(t);
            if (a.ok && kind > DQ_BF16) c.refuse(name, "float32, float16 or bfloat16 is wanted");
            if (a.ok && !c.truth(t, a.lib->is_contiguous)) c.refuse(name, "not contiguous");
            c.here(t, name);
            type.push_back(kind);
            len.push_back(c.number(t, a.lib->numel));
            data.push_back(a.data_of<void>(t));
        }
        Py_DECREF(items);
    }
    int32_t size() const { return static_cast<int32_t>(data.size()); }
};

// (grads, norm, workspace, device, stream)
PyObject* py_grad_norm(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 5);
    checker c(a, a.ok ? PyLong_AsLongLong(args[3]) : 0);
    tensor_list grads;
    grads.take(c, "grads");
    auto* norm = c.array<float>("norm", KIND_F32, 1);
    void* workspace = c.workspace(a.ok ? a.lib->dq_clip_workspace_bytes() : 0);
    a.object();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_grad_norm(grads.data.data(), grads.len.data(), grads.type.data(), grads.size(), norm, workspace, stream); });
}

// (grads, out or None, max_norm, norm, workspace, device, stream)
PyObject* py_clip_grads(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 7);
    checker c(a, a.ok ? PyLong_AsLongLong(args[5]) : 0);
    tensor_list grads, out;
    grads.take(c, "grads");
    const bool in_place = a.ok && args[1] == Py_None;
    if (in_place)
        a.object();
    else
        out.take(c, "out");
    if (a.ok && !in_place && (out.len != grads.len || out.type != grads.type)) c.refuse("out", "the gradients' sizes and types are wanted");
    const double max_norm = a.as_double();
    auto* norm = c.array<float>("norm", KIND_F32, 1);
    void* workspace = c.workspace(a.ok ? a.lib->dq_clip_workspace_bytes() : 0);
    a.object();
    void* stream = a.address();
    return status_of(a, [&] {
        return a.lib->dq_clip_grads(grads.data.data(), in_place ? grads.data.data() : out.data.data(), grads.len.data(), grads.type.data(), grads.size(), max_norm, norm,
                                    workspace, stream);
    });
}

// (plan, its lengths' address, grads, max_norm, norm, row, its length, workspace, device, stream)
PyObject* py_clip_gather(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 10);
    checker c(a, a.ok ? PyLong_AsLongLong(args[8]) : 0);
    const auto* plan = static_cast<const dq_plan_t*>(a.address());
    const auto* lens = static_cast<const int64_t*>(a.address());
    tensor_list grads;
    grads.take(c, "grads");
    if (a.ok && grads.size() != a.lib->dq_plan_num_segments(plan)) c.refuse("grads", "the plan has another number of tensors");
    for (int32_t l = 0; l < grads.size() && a.ok; ++l)
        if (grads.len[l] != lens[l]) c.refuse("grads", "the plan has another length for a tensor");
    const double max_norm = a.as_double();
    auto* norm = c.array<float>("norm", KIND_F32, 1);
    const int64_t length = a.ok ? PyLong_AsLongLong(args[6]) : 0;
    auto* row = c.array<float>("row", KIND_F32, length);
    a.object();
    void* workspace = c.workspace(a.ok ? a.lib->dq_clip_workspace_bytes() : 0);
    a.object();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_clip_gather(plan, grads.data.data(), grads.type.data(), max_norm, norm, row, workspace, stream); });
}

// (norms, M, n_seg, max_norm, total, out, workspace, device, stream)
PyObject* py_clip_norms(PyObject* module, args_t args, Py_ssize_t n)
{
    taker a(module, args, n, 9);
    checker c(a, a.ok ? PyLong_AsLongLong(args[7]) : 0);
    const int64_t M = a.ok ? PyLong_AsLongLong(args[1]) : 0, n_seg = a.ok ? PyLong_AsLongLong(args[2]) : 0;
    const auto* norms = c.array<const float>("norms", KIND_F32, M * n_seg);
    a.object();
    a.object();
    const double max_norm = a.as_double();
    auto* total = c.array<float>("total", KIND_F32, M);
    auto* out = c.array<float>("out", KIND_F32, M * n_seg);
    void* workspace = c.workspace(a.ok && M <= DQ_MAX_WORKERS ? a.lib->dq_clip_norms_workspace_bytes(static_cast<int>(M), n_seg) : 0);
    a.object();
    void* stream = a.address();
    return status_of(a, [&] { return a.lib->dq_clip_norms(norms, M > DQ_MAX_WORKERS ? -1 : static_cast<int>(M), n_seg, max_norm, total, out, workspace, stream); });
}

// (float32, float16, bfloat16, int64): torch's types
PyObject* py_set_types(PyObject* module, args_t args, Py_ssize_t n)
{
    state* lib = state_of(module);
    if (n != KINDS) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", static_cast<Py_ssize_t>(KINDS), n);
        return nullptr;
    }
    for (int k = 0; k < KINDS; ++k) {
        Py_INCREF(args[k]);
        Py_XSETREF(lib->types[k], args[k]);
    }
    Py_RETURN_NONE;
}

// ({name: address} of `functions`): the library that the other calls go to.
PyObject* py_bind(PyObject* module, PyObject* addresses)
{
    state* lib = state_of(module);
    if (!PyDict_Check(addresses)) {
        PyErr_SetString(PyExc_TypeError, "a dict of addresses");
        return nullptr;
    }
    lib->bound = false;
    const auto take = [&](const char* name) -> void* {
        PyObject* at = PyDict_GetItemString(addresses, name); // borrowed
        void* fn = at ? PyLong_AsVoidPtr(at) : nullptr;
        if (!fn && !PyErr_Occurred()) PyErr_Format(PyExc_ImportError, "%s: not in this library", name);
        return fn;
    };
#define X(fn)                                               \
    lib->fn = reinterpret_cast<decltype(&::fn)>(take(#fn)); \
    if (!lib->fn) return nullptr;
    DQ_FUNCTIONS(X)
#undef X
    lib->bound = true;
    Py_RETURN_NONE;
}

#define DQ_METHOD(name, fn) { name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(fn)), METH_FASTCALL, nullptr }
PyMethodDef methods[] = {
    { "bind", py_bind, METH_O, nullptr },
    DQ_METHOD("norm", py_norm),
    DQ_METHOD("quantize_pack", py_quantize_pack),
    DQ_METHOD("quantize_pack_v", py_quantize_pack_v),
    DQ_METHOD("norm_quantize_pack", py_norm_quantize_pack),
    DQ_METHOD("norm_bracket", py_norm_bracket),
    DQ_METHOD("bracketed", py_bracketed),
    DQ_METHOD("reduce", py_reduce),
    DQ_METHOD("reduce_update", py_reduce_update),
    DQ_METHOD("reduce_v", py_reduce_v),
    DQ_METHOD("reduce_update_v", py_reduce_update_v),
    DQ_METHOD("sign_pack", py_sign_pack),
    DQ_METHOD("sign_reduce", py_sign_reduce),
    DQ_METHOD("select_bits", py_select_bits),
    DQ_METHOD("packed_bytes", py_packed_bytes),
    DQ_METHOD("token_logprob", py_token_logprob),
    DQ_METHOD("token_logprob_backward", py_token_logprob_backward),
    DQ_METHOD("policy_loss", py_policy_loss),
    DQ_METHOD("preference_loss", py_preference_loss),
    DQ_METHOD("grad_norm", py_grad_norm),
    DQ_METHOD("clip_grads", py_clip_grads),
    DQ_METHOD("clip_gather", py_clip_gather),
    DQ_METHOD("clip_norms", py_clip_norms),
    DQ_METHOD("set_types", py_set_types),
    { nullptr, nullptr, 0, nullptr },
};

template <typename T>
T same(T value)
{
    return value;
}
uint64_t number(void* address) { return reinterpret_cast<uint64_t>(address); }

// ctypes.PYFUNCTYPE(result, argument)(fn); nullptr, with an exception set, if that fails or one is set already
template <typename F>
PyObject* returning(PyObject* ctypes, const char* result, const char* argument, F* fn)
{
    if (PyErr_Occurred()) return nullptr;
    PyObject* result_type = PyObject_GetAttrString(ctypes, result);
    PyObject* argument_type = result_type ? PyObject_GetAttrString(ctypes, argument) : nullptr;
    PyObject* type = argument_type ? PyObject_CallMethod(ctypes, "PYFUNCTYPE", "OO", result_type, argument_type) : nullptr;
    PyObject* made = type ? PyObject_CallFunction(type, "K", static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(fn))) : nullptr;
    Py_XDECREF(type);
    Py_XDECREF(argument_type);
    Py_XDECREF(result_type);
    return made;
}

int fill(PyObject* module)
{
    state* lib = state_of(module);
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    if (!ctypes) return -1;
    lib->convert[INT32] = returning(ctypes, "c_int32", "c_int32", &same<int32_t>);
    lib->convert[UINT32] = returning(ctypes, "c_uint32", "c_uint32", &same<uint32_t>);
    lib->convert[INT64] = returning(ctypes, "c_int64", "c_int64", &same<int64_t>);
    lib->convert[UINT64] = returning(ctypes, "c_uint64", "c_uint64", &same<uint64_t>);
    lib->convert[ADDRESS] = returning(ctypes, "c_uint64", "c_void_p", &number);
    lib->convert[FLOAT32] = returning(ctypes, "c_float", "c_float", &same<float>);
    lib->convert[FLOAT64] = returning(ctypes, "c_double", "c_double", &same<double>);
    Py_DECREF(ctypes);
    for (const PyObject* convert : lib->convert)
        if (!convert) return -1;
    lib->data_ptr = PyUnicode_InternFromString("data_ptr");
    lib->stride = PyUnicode_InternFromString("stride");
    lib->size = PyUnicode_InternFromString("size");
    lib->shape = PyUnicode_InternFromString("shape");
    lib->zero = PyLong_FromLong(0);
    lib->dtype = PyUnicode_InternFromString("dtype");
    lib->numel = PyUnicode_InternFromString("numel");
    lib->element_size = PyUnicode_InternFromString("element_size");
    lib->get_device = PyUnicode_InternFromString("get_device");
    lib->is_contiguous = PyUnicode_InternFromString("is_contiguous");
    if (!lib->data_ptr || !lib->stride || !lib->size || !lib->shape || !lib->zero || !lib->dtype || !lib->numel || !lib->element_size || !lib->get_device ||
        !lib->is_contiguous)
        return -1;
    static const char* const functions[] = {
#define X(fn) #fn,
        DQ_FUNCTIONS(X)
#undef X
    };
    PyObject* names = PyList_New(0);
    if (!names) return -1;
    for (const char* function : functions) {
        PyObject* name = PyUnicode_FromString(function);
        const bool added = name && PyList_Append(names, name) == 0;
        Py_XDECREF(name);
        if (!added) {
            Py_DECREF(names);
            return -1;
        }
    }
    if (PyModule_AddObject(module, "functions", names) != 0) {
        Py_DECREF(names);
        return -1;
    }
    return 0;
}

int visit_state(PyObject* module, visitproc visit, void* arg)
{
    if (state* lib = state_of(module)) {
        for (PyObject* convert : lib->convert) Py_VISIT(convert);
        for (PyObject* type : lib->types) Py_VISIT(type);
    }
    return 0;
}
int clear_state(PyObject* module)
{
    if (state* lib = state_of(module)) {
        for (PyObject*& convert : lib->convert) Py_CLEAR(convert);
        Py_CLEAR(lib->data_ptr);
        Py_CLEAR(lib->stride);
        Py_CLEAR(lib->size);
        Py_CLEAR(lib->shape);
        Py_CLEAR(lib->zero);
        Py_CLEAR(lib->dtype);
        Py_CLEAR(lib->numel);
        Py_CLEAR(lib->element_size);
        Py_CLEAR(lib->get_device);
        Py_CLEAR(lib->is_contiguous);
        for (PyObject*& type : lib->types) Py_CLEAR(type);
        lib->bound = false;
    }
    return 0;
}
void free_state(void* module) { clear_state(static_cast<PyObject*>(module)); }

PyModuleDef_Slot slots[] = { { Py_mod_exec, reinterpret_cast<void*>(fill) }, { 0, nullptr } };
PyModuleDef definition = { PyModuleDef_HEAD_INIT, "_dqcall", "Calls of libdq.so's per-iteration entry points.", sizeof(state), methods, slots, visit_state, clear_state, free_state };

} // namespace

PyMODINIT_FUNC PyInit__dqcall(void) { return PyModuleDef_Init(&definition); }
