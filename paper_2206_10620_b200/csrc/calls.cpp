// CPython extension with the enqueueing calls of the C ABI: argument marshalling only.  A layer of a
// small problem runs in a few microseconds, of which ctypes would take more than one.
#define PY_SSIZE_T_CLEAN
#define Py_LIMITED_API 0x030A0000
#include <Python.h>

#include "adapters.h"
#include "attention.h"
#include "blockgemm.h"
#include "dwconv.h"
#include "logprobs.h"

static decltype(&xgen_patconv_run) p_conv;
static decltype(&xgen_patconv_run_fused) p_fused;
static decltype(&xgen_blockgemm_run) p_gemm;
static decltype(&xgen_dwconv_run) p_dw;
static decltype(&xgen_adapters_run) p_adapters;
static decltype(&xgen_logprobs_run) p_logprobs;
static decltype(&xgen_attention_append) p_append;
static decltype(&xgen_attention_read) p_read;
static decltype(&xgen_attention_run) p_attend;

// Addresses are ints; None is the null pointer.
static void *ptr(PyObject *o) { return o == Py_None ? nullptr : PyLong_AsVoidPtr(o); }
static int64_t i64(PyObject *o) { return PyLong_AsLongLong(o); }
static int32_t i32(PyObject *o) { return (int32_t)PyLong_AsLong(o); }
static bool count(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
    return false;
}
static PyObject *status(xgen_status s) { return PyLong_FromLong((long)s); }

// bind(addresses of run, run_fused, blockgemm_run, dwconv_run, adapters_run, logprobs_run, attention_append, _read, _run)
static PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 9)) return nullptr;
    p_conv = reinterpret_cast<decltype(p_conv)>(ptr(a[0]));
    p_fused = reinterpret_cast<decltype(p_fused)>(ptr(a[1]));
    p_gemm = reinterpret_cast<decltype(p_gemm)>(ptr(a[2]));
    p_dw = reinterpret_cast<decltype(p_dw)>(ptr(a[3]));
    p_adapters = reinterpret_cast<decltype(p_adapters)>(ptr(a[4]));
    p_logprobs = reinterpret_cast<decltype(p_logprobs)>(ptr(a[5]));
    p_append = reinterpret_cast<decltype(p_append)>(ptr(a[6]));
    p_read = reinterpret_cast<decltype(p_read)>(ptr(a[7]));
    p_attend = reinterpret_cast<decltype(p_attend)>(ptr(a[8]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// conv / dw(handle, x, n, h, w, bias, relu, y, stream)
template <bool DW> static PyObject *run(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 9)) return nullptr;
    void *const h = ptr(a[0]), *const x = ptr(a[1]), *const bias = ptr(a[5]), *const y = ptr(a[7]), *const st = ptr(a[8]);
    const int32_t in = i32(a[2]), ih = i32(a[3]), iw = i32(a[4]), relu = PyObject_IsTrue(a[6]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    if (DW) s = p_dw(static_cast<const xgen_dwconv_packed *>(h), x, in, ih, iw, bias, relu, y, st);
    else s = p_conv(static_cast<const xgen_patconv_packed *>(h), x, in, ih, iw, bias, relu, y, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// fused(handle, x, n, h, w, bias, y, stream, relu, pool, residual, scale, zero point)
static PyObject *fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 13)) return nullptr;
    void *const h = ptr(a[0]), *const x = ptr(a[1]), *const bias = ptr(a[5]), *const y = ptr(a[6]), *const st = ptr(a[7]);
    const int32_t in = i32(a[2]), ih = i32(a[3]), iw = i32(a[4]);
    xgen_patconv_epilogue ep;
    ep.relu = PyObject_IsTrue(a[8]);
    ep.pool = i32(a[9]);
    ep.residual_dev = ptr(a[10]);
    ep.requant_scale_dev = static_cast<const float *>(ptr(a[11]));
    ep.requant_zero_point = i32(a[12]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_fused(static_cast<const xgen_patconv_packed *>(h), x, in, ih, iw, bias, &ep, y, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// gemm(handle, x, rows, bias, relu, y, stream)
static PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 7)) return nullptr;
    void *const h = ptr(a[0]), *const x = ptr(a[1]), *const bias = ptr(a[3]), *const y = ptr(a[5]), *const st = ptr(a[6]);
    const int64_t m = PyLong_AsLongLong(a[2]);
    const int32_t relu = PyObject_IsTrue(a[4]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_gemm(static_cast<const xgen_blockgemm_packed *>(h), x, m, bias, relu, y, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// adapters(handle, x, rows, x stride, row starts, adapters, requests, y, y stride, out, out stride, stream)
static PyObject *adapters(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 12)) return nullptr;
    void *const h = ptr(a[0]), *const x = ptr(a[1]), *const start = ptr(a[4]), *const which = ptr(a[5]), *const y = ptr(a[7]),
               *const out = ptr(a[9]), *const st = ptr(a[11]);
    const int64_t rows = i64(a[2]), xs = i64(a[3]), requests = i64(a[6]), ys = i64(a[8]), os = i64(a[10]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_adapters(static_cast<const xgen_adapters_packed *>(h), x, rows, xs, static_cast<const int32_t *>(start),
                   static_cast<const int32_t *>(which), requests, y, ys, out, os, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// logprobs(handle, x, rows, row stride, tokens, logprob, entropy, top, top_logprob, stream)
static PyObject *logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 10)) return nullptr;
    void *const h = ptr(a[0]), *const x = ptr(a[1]), *const token = ptr(a[4]), *const logprob = ptr(a[5]), *const entropy = ptr(a[6]),
               *const top = ptr(a[7]), *const top_logprob = ptr(a[8]), *const st = ptr(a[9]);
    const int64_t rows = i64(a[2]), stride = i64(a[3]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_logprobs(static_cast<const xgen_logprobs_packed *>(h), x, rows, stride, static_cast<const int32_t *>(token),
                   static_cast<float *>(logprob), static_cast<float *>(entropy), static_cast<int32_t *>(top),
                   static_cast<float *>(top_logprob), st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// append(handle, k, v, stride, batch, cache, stream)
static PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 7)) return nullptr;
    void *const h = ptr(a[0]), *const k = ptr(a[1]), *const v = ptr(a[2]), *const batch = ptr(a[4]), *const cache = ptr(a[5]), *const st = ptr(a[6]);
    const int64_t stride = i64(a[3]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_append(static_cast<const xgen_attention_packed *>(h), k, v, stride, static_cast<const xgen_attention_batch *>(batch),
                 static_cast<const xgen_attention_cache *>(cache), st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// read(handle, batch, cache, type, k, v, stride, stream)
static PyObject *read_back(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 8)) return nullptr;
    void *const h = ptr(a[0]), *const batch = ptr(a[1]), *const cache = ptr(a[2]), *const k = ptr(a[4]), *const v = ptr(a[5]), *const st = ptr(a[7]);
    const int32_t type = i32(a[3]);
    const int64_t stride = i64(a[6]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_read(static_cast<const xgen_attention_packed *>(h), static_cast<const xgen_attention_batch *>(batch),
               static_cast<const xgen_attention_cache *>(cache), static_cast<xgen_dtype>(type), k, v, stride, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

// attend(handle, q, q stride, batch, cache, y, y stride, workspace, stream)
static PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (!count(n, 9)) return nullptr;
    void *const h = ptr(a[0]), *const q = ptr(a[1]), *const batch = ptr(a[3]), *const cache = ptr(a[4]), *const y = ptr(a[5]),
               *const work = ptr(a[7]), *const st = ptr(a[8]);
    const int64_t qs = i64(a[2]), ys = i64(a[6]);
    if (PyErr_Occurred()) return nullptr;
    xgen_status s;
    Py_BEGIN_ALLOW_THREADS
    s = p_attend(static_cast<const xgen_attention_packed *>(h), q, qs, static_cast<const xgen_attention_batch *>(batch),
                 static_cast<const xgen_attention_cache *>(cache), y, ys, work, st);
    Py_END_ALLOW_THREADS
    return status(s);
}

template <typename F> static PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }
static PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},   {"conv", fast(run<false>), METH_FASTCALL, nullptr},
    {"fused", fast(fused), METH_FASTCALL, nullptr}, {"gemm", fast(gemm), METH_FASTCALL, nullptr},
    {"dw", fast(run<true>), METH_FASTCALL, nullptr}, {"adapters", fast(adapters), METH_FASTCALL, nullptr},
    {"logprobs", fast(logprobs), METH_FASTCALL, nullptr}, {"append", fast(append), METH_FASTCALL, nullptr},
    {"read", fast(read_back), METH_FASTCALL, nullptr}, {"attend", fast(attend), METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
// What the extension was made from: build.py looks for it in the file.
extern "C" __attribute__((used, visibility("default"))) const char xgen_calls_tag[] = XGEN_CALLS_TAG;
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
