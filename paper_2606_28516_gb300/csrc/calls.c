/* The calls of the 8-bit and few-token operators whose time the host bounds, as Python functions of integers (addresses,
 * sizes, codes; None for a null pointer). ctypes took 0.6 us for the arguments of such a call and as much again for the
 * epilogue's structure, of 4 to 6 us for the whole call. The functions are libclearmoe's, by the addresses that bind()
 * got; each returns its clearmoe_status and runs without the interpreter's lock. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "clearmoe.h"

static int (*g_quantize_rows)(const void*, int32_t, int64_t, const int32_t*, const clearmoe_fp8*, void*);
static int (*g_gemm)(const clearmoe_fp8*, const clearmoe_fp8*, const clearmoe_fp8_epilogue*, void*, int32_t, int64_t, void*);
static int (*g_gemm_fp8)(const clearmoe_fp8*, const clearmoe_fp8*, const clearmoe_fp8_epilogue*, const clearmoe_fp8*, void*);
static int (*g_few)(clearmoe_layer*, const void*, int64_t, const clearmoe_ffn_weights*, void*, void*);
static int (*g_fp8)(clearmoe_layer*, const void*, int64_t, const clearmoe_ffn_weights*, void*, void*);

/* The arguments as integers; 0 with an exception set when there are not n of them or one is no integer. */
static int integers(PyObject* const* args, Py_ssize_t got, Py_ssize_t n, int64_t* v) {
    if (got != n) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", n, got);
        return 0;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (args[i] == Py_None) {
            v[i] = 0;
            continue;
        }
        v[i] = (int64_t)PyLong_AsUnsignedLongLongMask(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return 0;
    }
    return 1;
}
#define PTR(i) ((void*)(intptr_t)v[i])

static PyObject* bind(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[5];
    (void)self;
    if (!integers(args, n, 5, v)) return NULL;
    *(void**)&g_quantize_rows = PTR(0);
    *(void**)&g_gemm = PTR(1);
    *(void**)&g_gemm_fp8 = PTR(2);
    *(void**)&g_few = PTR(3);
    *(void**)&g_fp8 = PTR(4);
    Py_RETURN_NONE;
}

/* x, dtype, ld, gather, out, stream */
static PyObject* quantize_rows(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[6];
    int rc;
    (void)self;
    if (!integers(args, n, 6, v)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = g_quantize_rows(PTR(0), (int32_t)v[1], v[2], PTR(3), PTR(4), PTR(5));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A, W, bias, its dtype, act, status, out, its dtype, ldo, stream */
static PyObject* gemm(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[10];
    int rc;
    (void)self;
    if (!integers(args, n, 10, v)) return NULL;
    const clearmoe_fp8_epilogue epi = {PTR(2), (int32_t)v[3], (int32_t)v[4], PTR(5)};
    Py_BEGIN_ALLOW_THREADS
    rc = g_gemm(PTR(0), PTR(1), &epi, PTR(6), (int32_t)v[7], v[8], PTR(9));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A, W, bias, its dtype, act, status, out, stream */
static PyObject* gemm_fp8(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[8];
    int rc;
    (void)self;
    if (!integers(args, n, 8, v)) return NULL;
    const clearmoe_fp8_epilogue epi = {PTR(2), (int32_t)v[3], (int32_t)v[4], PTR(5)};
    Py_BEGIN_ALLOW_THREADS
    rc = g_gemm_fp8(PTR(0), PTR(1), &epi, PTR(6), PTR(7));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* layer, x, T, weights, out, stream */
static PyObject* ffn(PyObject* const* args, Py_ssize_t n,
                     int (*fn)(clearmoe_layer*, const void*, int64_t, const clearmoe_ffn_weights*, void*, void*)) {
    int64_t v[6];
    int rc;
    if (!integers(args, n, 6, v)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(PTR(0), PTR(1), v[2], PTR(3), PTR(4), PTR(5));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
static PyObject* ffn_few(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    return ffn(args, n, g_few);
}
static PyObject* ffn_fp8(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    return ffn(args, n, g_fp8);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind),    METHOD(quantize_rows), METHOD(gemm), METHOD(gemm_fp8),
                                METHOD(ffn_few), METHOD(ffn_fp8),       {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }
