/*
 * marshal.c -- the Python side of the entry points that a decoding step calls between its int8 products.
 *
 * The same calls as through ctypes: arguments are taken apart here, handed to the C ABI of libabft.so, and its return code comes back.
 * A call's 17 to 25 arguments, its stream's handle with them, take 1.5 to 2.05 us by ctypes and 0.5 to 0.6 here, where the launch
 * itself takes 3.3: what a program waits for that calls many small layers and records no graph (1 x 4096 normed and quantised: 5.5 us a
 * call before, 4.2 now).  Pointers are tensors (their data_ptr()), integers or None; a fault descriptor is the ctypes
 * structure, read through the buffer protocol.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/abft.h"

static PyObject *s_data_ptr;

/* addresses of the entry points, handed over once by the binding that has loaded the library */
static int (*f_add)(int, int, int, const void *, int64_t, const float *, const void *, int64_t, int, const float *, const float *, int, const void *,
                    int64_t, void *, int64_t, int, int, const void *, void *, size_t, uint32_t *, abft_report_t *, const abft_fault_t *, void *);
static int (*f_linear_add)(int, int, int, const void *, int64_t, int, const void *, int64_t, int, const float *, const float *, int, const void *,
                           int64_t, void *, int64_t, int, const void *, void *, size_t, uint32_t *, abft_report_t *, const abft_fault_t *, void *);
static int (*f_gated)(int, int, int, const void *, int64_t, const float *, const void *, int64_t, int, const float *, const float *, int, void *,
                      int64_t, int, int, const void *, void *, size_t, uint32_t *, abft_report_t *, const abft_fault_t *, void *);
static int (*f_linear_gated)(int, int, int, const void *, int64_t, int, const void *, int64_t, int, const float *, const float *, int, void *,
                             int64_t, int, const void *, void *, size_t, uint32_t *, abft_report_t *, const abft_fault_t *, void *);
static int (*f_norm)(int, int, const void *, int64_t, int, const float *, float, const void *, int64_t, void *, int64_t, void *, int64_t, void *,
                     int64_t, float *, void *);

/* The conversions.  After an error they return 0 with the exception set, and convert nothing more; callers look for it once, before
 * the call. */
static int64_t as_i64(PyObject *o) { return PyErr_Occurred() ? 0 : PyLong_AsLongLong(o); }
static int as_int(PyObject *o) {
    const int64_t v = as_i64(o);
    if (v != (int)v) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_OverflowError, "an argument does not fit 32 bits");
        return 0;
    }
    return (int)v;
}
static void *as_ptr(PyObject *o) {
    if (o == Py_None || PyErr_Occurred()) return NULL;
    if (PyLong_Check(o)) return PyLong_AsVoidPtr(o);
    PyObject *const p = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!p) return NULL;
    void *const v = PyLong_AsVoidPtr(p);
    Py_DECREF(p);
    return v;
}
/* (the structure is read during the call only, and the caller holds it) */
static const abft_fault_t *as_fault(PyObject *o) {
    Py_buffer b;
    if (o == Py_None || PyErr_Occurred() || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) return NULL;
    const abft_fault_t *const f = (size_t)b.len == sizeof *f ? (const abft_fault_t *)b.buf : NULL;
    if (!f) PyErr_SetString(PyExc_TypeError, "inject has to be a Fault");
    PyBuffer_Release(&b);
    return f;
}
static int wanted(Py_ssize_t got, Py_ssize_t want) {
    if (got == want && f_norm) return 1;
    if (!f_norm) {
        PyErr_SetString(PyExc_RuntimeError, "bind() comes first");
        return 0;
    }
    PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
    return 0;
}
#define I(k) as_int(a[k])
#define Q(k) as_i64(a[k])
#define P(k) as_ptr(a[k])
/* the call itself without the interpreter's lock: a launch may wait for room in its queue */
#define CALL(expr)                              \
    do {                                        \
        int rc;                                 \
        if (PyErr_Occurred()) return NULL;      \
        Py_BEGIN_ALLOW_THREADS rc = (expr);     \
        Py_END_ALLOW_THREADS                    \
        return PyLong_FromLong(rc);             \
    } while (0)

static PyObject *gemm_scaled_add(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!wanted(n, 25)) return NULL;
    const int M = I(0), N = I(1), K = I(2), layout = I(8), act = I(11), dt = I(16), mode = I(17);
    const int64_t lda = Q(4), ldb = Q(7), ldr = Q(13), ldc = Q(15), bytes = Q(20);
    void *const A = P(3), *const rs = P(5), *const B = P(6), *const cs = P(9), *const bias = P(10), *const R = P(12), *const C = P(14), *const beta = P(18),
               *const ws = P(19), *const flag = P(21), *const rep = P(22), *const st = P(24);
    const abft_fault_t *const inject = as_fault(a[23]);
    CALL(f_add(M, N, K, A, lda, rs, B, ldb, layout, cs, bias, act, R, ldr, C, ldc, dt, mode, beta, ws, (size_t)bytes, flag, rep, inject, st));
}
static PyObject *linear_scaled_add(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!wanted(n, 24)) return NULL;
    const int M = I(0), N = I(1), K = I(2), dt = I(5), layout = I(8), act = I(11), mode = I(16);
    const int64_t ldx = Q(4), ldb = Q(7), ldr = Q(13), ldc = Q(15), bytes = Q(19);
    void *const X = P(3), *const B = P(6), *const cs = P(9), *const bias = P(10), *const R = P(12), *const C = P(14), *const beta = P(17), *const ws = P(18),
               *const flag = P(20), *const rep = P(21), *const st = P(23);
    const abft_fault_t *const inject = as_fault(a[22]);
    CALL(f_linear_add(M, N, K, X, ldx, dt, B, ldb, layout, cs, bias, act, R, ldr, C, ldc, mode, beta, ws, (size_t)bytes, flag, rep, inject, st));
}
static PyObject *gemm_gated(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!wanted(n, 23)) return NULL;
    const int M = I(0), N = I(1), K = I(2), layout = I(8), act = I(11), dt = I(14), mode = I(15);
    const int64_t lda = Q(4), ldb = Q(7), ldc = Q(13), bytes = Q(18);
    void *const A = P(3), *const rs = P(5), *const B = P(6), *const cs = P(9), *const bias = P(10), *const C = P(12), *const beta = P(16), *const ws = P(17),
               *const flag = P(19), *const rep = P(20), *const st = P(22);
    const abft_fault_t *const inject = as_fault(a[21]);
    CALL(f_gated(M, N, K, A, lda, rs, B, ldb, layout, cs, bias, act, C, ldc, dt, mode, beta, ws, (size_t)bytes, flag, rep, inject, st));
}
static PyObject *linear_gated(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!wanted(n, 22)) return NULL;
    const int M = I(0), N = I(1), K = I(2), dt = I(5), layout = I(8), act = I(11), mode = I(14);
    const int64_t ldx = Q(4), ldb = Q(7), ldc = Q(13), bytes = Q(17);
    void *const X = P(3), *const B = P(6), *const cs = P(9), *const bias = P(10), *const C = P(12), *const beta = P(15), *const ws = P(16), *const flag = P(18),
               *const rep = P(19), *const st = P(21);
    const abft_fault_t *const inject = as_fault(a[20]);
    CALL(f_linear_gated(M, N, K, X, ldx, dt, B, ldb, layout, cs, bias, act, C, ldc, mode, beta, ws, (size_t)bytes, flag, rep, inject, st));
}
static PyObject *rms_norm(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (!wanted(n, 17)) return NULL;
    const int M = I(0), K = I(1), dt = I(4);
    const int64_t ldx = Q(3), ldr = Q(8), lds = Q(10), ldy = Q(12), ldq = Q(14);
    const double eps = PyErr_Occurred() ? 0 : PyFloat_AsDouble(a[6]);
    void *const X = P(2), *const w = P(5), *const R = P(7), *const S = P(9), *const Y = P(11), *const q = P(13), *const scale = P(15), *const st = P(16);
    CALL(f_norm(M, K, X, ldx, dt, w, (float)eps, R, ldr, S, lds, Y, ldy, q, ldq, scale, st));
}
/* bind(gemm_scaled_add, linear_scaled_add, gemm_gated, linear_gated, rms_norm): their addresses */
static PyObject *bind(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "5 addresses");
        return NULL;
    }
    *(void **)&f_add = P(0);
    *(void **)&f_linear_add = P(1);
    *(void **)&f_gated = P(2);
    *(void **)&f_linear_gated = P(3);
    *(void **)&f_norm = P(4);
    if (PyErr_Occurred()) return NULL;
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(gemm_scaled_add), METHOD(linear_scaled_add), METHOD(gemm_gated), METHOD(linear_gated), METHOD(rms_norm), METHOD(bind), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    return s_data_ptr ? PyModule_Create(&module) : NULL;
}
