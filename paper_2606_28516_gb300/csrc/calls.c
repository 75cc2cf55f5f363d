/* The calls of the 8-bit and few-token operators whose time the host bounds. ctypes took 0.6 us for the arguments of such a
 * call and as much again for the epilogue's structure, and the looks at tensors in Python as much as that, of 4 to 6 us
 * for the whole call.
 *
 * quantize_rows, gemm, gemm_fp8, ffn_few, ffn_fp8 take integers (addresses, sizes, codes; None for a null pointer); the
 * same names with _t take the tensors and return None, having called nothing, for an argument that is not as it should
 * be, which the Python side then looks at and refuses. Otherwise each returns the clearmoe_status of libclearmoe's
 * function, got by bind(), and runs it without the interpreter's lock. */
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

/* ---- from tensors ---- */
static PyObject *s_is_cuda, *s_shape, *s_stride, *s_data_ptr, *s_dtype, *s_is_contiguous, *s_numel, *s_cuda_stream;
static PyObject *g_bf16, *g_f32, *g_i32, *g_get_device, *g_raw_stream; /* torch's dtypes; the current device; its current stream */

/* bfloat16, float32, int32, a function giving the current device, one giving a device's current stream */
static PyObject* bind_torch(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    PyObject** to[5] = {&g_bf16, &g_f32, &g_i32, &g_get_device, &g_raw_stream};
    (void)self;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments expected, got %zd", n);
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(args[i]);
        Py_XSETREF(*to[i], args[i]);
    }
    Py_RETURN_NONE;
}

/* Each of these: 0 for an argument that is not as it should be, with no exception left. */
static int yes(PyObject* o) { /* takes the reference */
    const int r = o == Py_True;
    if (!o) PyErr_Clear();
    Py_XDECREF(o);
    return r;
}
static int integer(PyObject* o, int64_t* v) { /* takes the reference */
    if (!o) {
        PyErr_Clear();
        return 0;
    }
    *v = (int64_t)PyLong_AsUnsignedLongLongMask(o);
    Py_DECREF(o);
    if (*v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return 0;
    }
    return 1;
}
static int pair(PyObject* o, int64_t* v) { /* takes the reference */
    int ok = o && PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2;
    for (int i = 0; i < 2 && ok; ++i) {
        Py_INCREF(PyTuple_GET_ITEM(o, i));
        ok = integer(PyTuple_GET_ITEM(o, i), v + i);
    }
    if (!o) PyErr_Clear();
    Py_XDECREF(o);
    return ok;
}
static int dtype_of(PyObject* t, int32_t* dt) {
    PyObject* o = PyObject_GetAttr(t, s_dtype);
    const int ok = o && (o == g_bf16 || o == g_f32);
    *dt = o == g_bf16 ? CLEARMOE_BF16 : CLEARMOE_F32;
    if (!o) PyErr_Clear();
    Py_XDECREF(o);
    return ok;
}
/* A [rows x cols] matrix of any row pitch. */
static int matrix(PyObject* t, int64_t rows, int64_t cols, int64_t* p, int32_t* dt, int64_t* ld) {
    int64_t shape[2], stride[2];
    if (!yes(PyObject_GetAttr(t, s_is_cuda)) || !pair(PyObject_GetAttr(t, s_shape), shape) || shape[0] != rows || shape[1] != cols ||
        !pair(PyObject_CallMethodNoArgs(t, s_stride), stride) || (cols > 1 && stride[1] != 1) || !dtype_of(t, dt))
        return 0;
    *ld = rows > 1 || stride[0] > cols ? stride[0] : cols;
    return integer(PyObject_CallMethodNoArgs(t, s_data_ptr), p);
}
/* A dense tensor, or None. */
static int dense(PyObject* t, int64_t* p) {
    *p = 0;
    return t == Py_None || (yes(PyObject_GetAttr(t, s_is_cuda)) && yes(PyObject_CallMethodNoArgs(t, s_is_contiguous)) &&
                            integer(PyObject_CallMethodNoArgs(t, s_data_ptr), p));
}
static int bias_of(PyObject* t, int64_t n, int64_t* p, int32_t* dt) {
    int64_t numel;
    *dt = CLEARMOE_F32;
    if (t == Py_None) {
        *p = 0;
        return 1;
    }
    return integer(PyObject_CallMethodNoArgs(t, s_numel), &numel) && numel == n && dense(t, p) && dtype_of(t, dt);
}
/* A status word, or None. */
static int status_of(PyObject* t, int64_t* p) {
    int64_t numel;
    *p = 0;
    if (t == Py_None) return 1;
    PyObject* o = PyObject_GetAttr(t, s_dtype);
    const int ok = o && o == g_i32;
    if (!o) PyErr_Clear();
    Py_XDECREF(o);
    return ok && integer(PyObject_CallMethodNoArgs(t, s_numel), &numel) && numel >= 1 && dense(t, p);
}
static int stream_of(PyObject* stream, int64_t* s) {
    if (!g_raw_stream) return 0;
    if (stream != Py_None) return integer(PyObject_GetAttr(stream, s_cuda_stream), s);
    PyObject* d = PyObject_CallNoArgs(g_get_device);
    PyObject* r = d ? PyObject_CallOneArg(g_raw_stream, d) : NULL;
    Py_XDECREF(d);
    return integer(r, s);
}
#define AT(x) ((void*)(intptr_t)(x))

/* x, rows, cols, out, stream */
static PyObject* quantize_rows_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[3], x, ld, s;
    int32_t dt;
    int rc;
    (void)self;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments expected, got %zd", n);
    if (!integers(args + 1, 3, 3, v)) return NULL;
    if (!stream_of(args[4], &s) || !matrix(args[0], v[0], v[1], &x, &dt, &ld)) Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    rc = g_quantize_rows(AT(x), dt, ld, NULL, PTR(2), AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A, W, rows, cols, act, bias, status, out, stream */
static PyObject* gemm_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[5], bias, status, out, ld, s;
    int32_t bias_dt, dt;
    int rc;
    (void)self;
    if (n != 9) return PyErr_Format(PyExc_TypeError, "9 arguments expected, got %zd", n);
    if (!integers(args, 5, 5, v)) return NULL;
    if (!stream_of(args[8], &s) || !bias_of(args[5], v[3], &bias, &bias_dt) || !status_of(args[6], &status) ||
        !matrix(args[7], v[2], v[3], &out, &dt, &ld))
        Py_RETURN_NONE;
    const clearmoe_fp8_epilogue epi = {AT(bias), bias_dt, (int32_t)v[4], AT(status)};
    Py_BEGIN_ALLOW_THREADS
    rc = g_gemm(PTR(0), PTR(1), &epi, AT(out), dt, ld, AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A dense [rows x cols] matrix of one dtype; rows < 0: any number, which it gets. */
static int tokens(PyObject* t, int64_t* rows, int64_t cols, int32_t dtype, int64_t* p) {
    int64_t shape[2];
    int32_t dt;
    if (t == Py_None || !pair(PyObject_GetAttr(t, s_shape), shape) || shape[1] != cols || (*rows >= 0 && shape[0] != *rows) ||
        !dtype_of(t, &dt) || dt != dtype)
        return 0;
    *rows = shape[0];
    return dense(t, p);
}

/* layer, weights (not null), x, out, stream */
static PyObject* ffn_t(PyObject* const* args, Py_ssize_t n,
                       int (*fn)(clearmoe_layer*, const void*, int64_t, const clearmoe_ffn_weights*, void*, void*)) {
    int64_t v[2], T = -1, x, out, s;
    int rc;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "5 arguments expected, got %zd", n);
    if (!integers(args, 2, 2, v)) return NULL;
    const clearmoe_ffn_weights* w = PTR(1);
    const int32_t dtype = w->dtype == CLEARMOE_F32 ? CLEARMOE_F32 : CLEARMOE_BF16; /* the layer's */
    if (!stream_of(args[4], &s) || !tokens(args[2], &T, w->W1.cols, dtype, &x) || !tokens(args[3], &T, w->W1.cols, dtype, &out))
        Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(PTR(0), AT(x), T, w, AT(out), AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
static PyObject* ffn_few_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    return ffn_t(args, n, g_few);
}
static PyObject* ffn_fp8_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    return ffn_t(args, n, g_fp8);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind),      METHOD(bind_torch),      METHOD(quantize_rows), METHOD(gemm),
                                METHOD(gemm_fp8),  METHOD(ffn_few),         METHOD(ffn_fp8),       METHOD(quantize_rows_t),
                                METHOD(gemm_t),    METHOD(ffn_few_t),       METHOD(ffn_fp8_t),     {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) {
    PyObject** names[] = {&s_is_cuda, &s_shape, &s_stride, &s_data_ptr, &s_dtype, &s_is_contiguous, &s_numel, &s_cuda_stream};
    const char* text[] = {"is_cuda", "shape", "stride", "data_ptr", "dtype", "is_contiguous", "numel", "cuda_stream"};
    for (int i = 0; i < 8; ++i)
        if (!(*names[i] = PyUnicode_InternFromString(text[i]))) return NULL;
    return PyModule_Create(&module);
}
