/* The calls of the 4-bit, 8-bit, norm and few-token operators whose time the host bounds. ctypes took 0.6 us for the arguments of such a
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
static PyObject *s_is_cuda, *s_shape, *s_stride, *s_data_ptr, *s_dtype, *s_is_contiguous, *s_numel, *s_cuda_stream, *s_device_index;
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
/* A tensor as its exchange capsule describes it (DLPack's structure, a public format): one call of torch's where its
 * attributes are five. */
struct exchanged {
    void* data;
    int32_t device_type, device_id, ndim;
    uint8_t code, bits;
    uint16_t lanes;
    int64_t* shape;
    int64_t* strides;
    uint64_t byte_offset;
};
enum { ON_CUDA = 2, CODE_INT = 0, CODE_FLOAT = 2, CODE_BFLOAT = 4 };
static PyObject* g_to_dlpack; /* torch's function, or NULL */

/* t as [rows x cols] (rows < 0: any number) on GPU `device` (negative: any): its shape, address, dtype and row pitch. 0 for
 * anything else, with no exception left. */
static int matrix_at(PyObject* t, int64_t rows, int64_t cols, int device, int64_t* shape, int64_t* p, int32_t* dt, int64_t* ld) {
    PyObject* capsule = g_to_dlpack ? PyObject_CallOneArg(g_to_dlpack, t) : NULL;
    const struct exchanged* x = capsule ? PyCapsule_GetPointer(capsule, "dltensor") : NULL;
    int ok = x && x->device_type == ON_CUDA && (device < 0 || x->device_id == device) && x->ndim == 2 && x->strides && x->lanes == 1 &&
             (rows < 0 || x->shape[0] == rows) && (cols < 0 || x->shape[1] == cols) && (x->shape[1] < 2 || x->strides[1] == 1) &&
             ((x->code == CODE_FLOAT && x->bits == 32) || (x->code == CODE_BFLOAT && x->bits == 16));
    if (ok) {
        shape[0] = x->shape[0];
        shape[1] = x->shape[1];
        *p = (int64_t)(intptr_t)x->data + (int64_t)x->byte_offset;
        *dt = x->bits == 16 ? CLEARMOE_BF16 : CLEARMOE_F32;
        *ld = shape[0] > 1 ? x->strides[0] : shape[1];
    }
    if (!x) PyErr_Clear();
    Py_XDECREF(capsule);
    return ok;
}

/* n elements in a row on GPU `device` (negative: any), or None: their address and dtype. 0 for anything else, with no
 * exception left. */
static int row_at(PyObject* t, int64_t n, int device, int64_t* p, int32_t* dt) {
    *p = 0;
    *dt = CLEARMOE_F32;
    if (t == Py_None) return 1;
    PyObject* capsule = g_to_dlpack ? PyObject_CallOneArg(g_to_dlpack, t) : NULL;
    const struct exchanged* x = capsule ? PyCapsule_GetPointer(capsule, "dltensor") : NULL;
    const int ok = x && x->device_type == ON_CUDA && (device < 0 || x->device_id == device) && x->ndim == 1 && x->strides && x->lanes == 1 &&
                   x->shape[0] == n && (n < 2 || x->strides[0] == 1) &&
                   ((x->code == CODE_FLOAT && x->bits == 32) || (x->code == CODE_BFLOAT && x->bits == 16));
    if (ok) {
        *p = (int64_t)(intptr_t)x->data + (int64_t)x->byte_offset;
        *dt = x->bits == 16 ? CLEARMOE_BF16 : CLEARMOE_F32;
    }
    if (!x) PyErr_Clear();
    Py_XDECREF(capsule);
    return ok;
}

/* A status word (dense int32, its first element) on GPU `device` (negative: any), or None: its address. 0 for anything else,
 * with no exception left. */
static int status_at(PyObject* t, int device, int64_t* p) {
    *p = 0;
    if (t == Py_None) return 1;
    PyObject* capsule = g_to_dlpack ? PyObject_CallOneArg(g_to_dlpack, t) : NULL;
    const struct exchanged* x = capsule ? PyCapsule_GetPointer(capsule, "dltensor") : NULL;
    int ok = x && x->device_type == ON_CUDA && (device < 0 || x->device_id == device) && x->code == CODE_INT && x->bits == 32 &&
             x->lanes == 1 && (x->ndim == 0 || x->strides);
    int64_t step = 1;
    for (int i = ok ? x->ndim - 1 : -1; i >= 0; --i) {
        ok = ok && x->shape[i] > 0 && (x->shape[i] == 1 || x->strides[i] == step);
        step *= x->shape[i];
    }
    if (ok) *p = (int64_t)(intptr_t)x->data + (int64_t)x->byte_offset;
    if (!x) PyErr_Clear();
    Py_XDECREF(capsule);
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

/* ---- 4-bit blocks and the norm ---- */
/* Matrices in blocks as the binding hands them over: the library's structure and, behind it, their GPU (-1: not known). */
struct placed_fp4 {
    clearmoe_fp4 m;
    int32_t device;
};
struct placed_fp8 {
    clearmoe_fp8 m;
    int32_t device;
};
static int here(int32_t at, int device) { return at < 0 || device < 0 || at == device; }
#define HERE4(p) here(((const struct placed_fp4*)(p))->device, device)
#define HERE8(p) here(((const struct placed_fp8*)(p))->device, device)
static int (*g_fp4_quantize)(const void*, int64_t, int32_t, int64_t, const int32_t*, const clearmoe_fp4*, void*);
static int (*g_fp4_gemm)(const clearmoe_fp4*, const clearmoe_fp4*, const clearmoe_fp8_epilogue*, void*, int32_t, int64_t, void*);
static int (*g_fp4_gemm_fp4)(const clearmoe_fp4*, const clearmoe_fp4*, const clearmoe_fp8_epilogue*, const clearmoe_fp4*, void*);
static int (*g_norm)(const clearmoe_norm*, void*, int32_t, int64_t, void*);
static int (*g_norm_fp8)(const clearmoe_norm*, const clearmoe_fp8*, void*);
static int (*g_norm_fp4)(const clearmoe_norm*, const clearmoe_fp4*, void*);

static PyObject* bind_fp4(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[6];
    (void)self;
    if (!integers(args, n, 6, v)) return NULL;
    *(void**)&g_fp4_quantize = PTR(0);
    *(void**)&g_fp4_gemm = PTR(1);
    *(void**)&g_fp4_gemm_fp4 = PTR(2);
    *(void**)&g_norm = PTR(3);
    *(void**)&g_norm_fp8 = PTR(4);
    *(void**)&g_norm_fp4 = PTR(5);
    Py_RETURN_NONE;
}

/* The stream's handle and its device (-1: not known). */
static int stream_and_device(PyObject* stream, int64_t* s, int* device) {
    int64_t d = -1;
    if (!g_raw_stream) return 0;
    if (stream != Py_None) {
        if (!integer(PyObject_GetAttr(stream, s_device_index), &d)) d = -1;
        *device = (int)d;
        return integer(PyObject_GetAttr(stream, s_cuda_stream), s);
    }
    PyObject* o = PyObject_CallNoArgs(g_get_device);
    PyObject* r = o ? PyObject_CallOneArg(g_raw_stream, o) : NULL;
    const int ok = integer(r, s) && integer(o, &d);
    if (!ok) PyErr_Clear();
    *device = (int)d;
    return ok;
}

/* torch's function that makes exchange capsules */
static PyObject* bind_dlpack(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    (void)self;
    if (n != 1) return PyErr_Format(PyExc_TypeError, "1 argument expected, got %zd", n);
    Py_INCREF(args[0]);
    Py_XSETREF(g_to_dlpack, args[0]);
    Py_RETURN_NONE;
}

/* x, out, stream */
static PyObject* fp4_quantize_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[1], shape[2], x, ld, s;
    int32_t dt;
    int rc, device;
    (void)self;
    if (n != 3) return PyErr_Format(PyExc_TypeError, "3 arguments expected, got %zd", n);
    if (!integers(args + 1, 1, 1, v)) return NULL;
    const clearmoe_fp4* out = PTR(0);
    if (!stream_and_device(args[2], &s, &device) || !HERE4(out) || !matrix_at(args[0], out->rows, out->cols, device, shape, &x, &dt, &ld)) Py_RETURN_NONE;
    Py_BEGIN_ALLOW_THREADS
    rc = g_fp4_quantize(AT(x), shape[0], dt, ld, NULL, out, AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* A, W, act, bias, status, out (a tensor, or the address of 4-bit blocks), stream */
static PyObject* fp4_gemm_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t v[3], shape[2], bias, status, out, ld = 0, s;
    int32_t bias_dt, dt = CLEARMOE_F32;
    int rc, device;
    (void)self;
    if (n != 7) return PyErr_Format(PyExc_TypeError, "7 arguments expected, got %zd", n);
    if (!integers(args, 3, 3, v)) return NULL;
    const clearmoe_fp4 *A = PTR(0), *W = PTR(1);
    if (!stream_and_device(args[6], &s, &device) || !HERE4(A) || !HERE4(W) || !row_at(args[3], W->rows, device, &bias, &bias_dt) ||
        !status_at(args[4], device, &status))
        Py_RETURN_NONE;
    const clearmoe_fp8_epilogue epi = {AT(bias), bias_dt, (int32_t)v[2], AT(status)};
    const int blocks = PyLong_Check(args[5]);
    if (blocks) {
        if (!integers(args + 5, 1, 1, &out)) return NULL;
        if (!HERE4(AT(out))) Py_RETURN_NONE;
    } else if (!matrix_at(args[5], A->rows, W->rows, device, shape, &out, &dt, &ld)) {
        Py_RETURN_NONE;
    }
    Py_BEGIN_ALLOW_THREADS
    rc = blocks ? g_fp4_gemm_fp4(A, W, &epi, AT(out), AT(s)) : g_fp4_gemm(A, W, &epi, AT(out), dt, ld, AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* x, residual, sum, weight (tensors or None), eps, bits (0: a tensor, 8 or 4: the address of blocks), out, stream */
static PyObject* rms_norm_t(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    int64_t shape[2], x, r = 0, sum = 0, w, out, ldo = 0, s, bits;
    int32_t dt, other, out_dt = CLEARMOE_F32;
    clearmoe_norm a = {0};
    int rc, device;
    (void)self;
    if (n != 8) return PyErr_Format(PyExc_TypeError, "8 arguments expected, got %zd", n);
    if (!integers(args + 5, 1, 1, &bits)) return NULL;
    a.eps = (float)PyFloat_AsDouble(args[4]);
    if (PyErr_Occurred()) return NULL;
    if (!stream_and_device(args[7], &s, &device) || !matrix_at(args[0], -1, -1, device, shape, &x, &dt, &a.ldx)) Py_RETURN_NONE;
    a.rows = shape[0];
    a.cols = shape[1];
    if ((args[1] != Py_None && (!matrix_at(args[1], a.rows, a.cols, device, shape, &r, &other, &a.ldr) || other != dt)) ||
        (args[2] != Py_None && (!matrix_at(args[2], a.rows, a.cols, device, shape, &sum, &other, &a.lds) || other != dt)) ||
        !row_at(args[3], a.cols, device, &w, &a.weight_dtype))
        Py_RETURN_NONE;
    if (bits) {
        if (!integers(args + 6, 1, 1, &out)) return NULL;
        if (!(bits == 8 ? HERE8(AT(out)) : HERE4(AT(out)))) Py_RETURN_NONE;
    } else if (!matrix_at(args[6], a.rows, a.cols, device, shape, &out, &out_dt, &ldo)) {
        Py_RETURN_NONE;
    }
    a.x = AT(x);
    a.residual = AT(r);
    a.sum = AT(sum);
    a.weight = AT(w);
    a.dtype = dt;
    Py_BEGIN_ALLOW_THREADS
    rc = bits == 8 ? g_norm_fp8(&a, AT(out), AT(s)) : bits == 4 ? g_norm_fp4(&a, AT(out), AT(s)) : g_norm(&a, AT(out), out_dt, ldo, AT(s));
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(bind),      METHOD(bind_torch),      METHOD(quantize_rows), METHOD(gemm),
                                METHOD(gemm_fp8),  METHOD(ffn_few),         METHOD(ffn_fp8),       METHOD(quantize_rows_t),
                                METHOD(gemm_t),    METHOD(ffn_few_t),       METHOD(ffn_fp8_t),
                                METHOD(bind_fp4),  METHOD(fp4_quantize_t),  METHOD(fp4_gemm_t),    METHOD(rms_norm_t),
                                METHOD(bind_dlpack),
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__calls(void) {
    PyObject** names[] = {&s_is_cuda, &s_shape, &s_stride, &s_data_ptr, &s_dtype, &s_is_contiguous, &s_numel, &s_cuda_stream,
                          &s_device_index};
    const char* text[] = {"is_cuda", "shape", "stride", "data_ptr", "dtype", "is_contiguous", "numel", "cuda_stream", "device_index"};
    for (int i = 0; i < 9; ++i)
        if (!(*names[i] = PyUnicode_InternFromString(text[i]))) return NULL;
    return PyModule_Create(&module);
}
