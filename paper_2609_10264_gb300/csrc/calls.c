/* The binding's calls of the client's attention, whose kernels for a few tokens take
 * less time than ctypes needs for a call's twenty arguments: a Python module that looks
 * at the tensors and calls libpvmvmd.so.  (One token rotated 3.7 us a call where 6.5
 * through ctypes, 8 appended 4.6 and 8.7, attention of 8 over 8 5.1 and 8.2, of which the
 * device takes the 5.1.)
 * Shapes, types and strides are checked here, everything else by the library. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include "pvmvmd.h"

static PyObject *s_is_cuda, *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_numel, *s_is_contiguous, *s_cuda_stream;
static PyObject *t_float[3];          /* bfloat16, float16, float32 */
static PyObject *t_int32, *t_uint32;  /* the latter may be None */
static PyObject *f_stream, *f_device; /* the current stream: f_stream(f_device()), or f_stream() */
static __typeof__(&pvmvmd_rope) f_rope;
static __typeof__(&pvmvmd_kv_append) f_append;
static __typeof__(&pvmvmd_paged_attention) f_attend;
static __typeof__(&pvmvmd_kv_evict) f_evict;

typedef struct {
    void *p;
    int64_t token, head;
} Rows;

static int on_device(PyObject *t, const char *name) {
    PyObject *c = PyObject_GetAttr(t, s_is_cuda);
    const int ok = c == Py_True;
    if (!c) PyErr_Clear();
    Py_XDECREF(c);
    if (!ok) PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
    return ok;
}
static int same_type(PyObject *t, const char *name, PyObject *want) {
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    const int ok = d == want;
    if (d && !ok) PyErr_Format(PyExc_TypeError, "%s must have dtype %S, got %S", name, want, d);
    Py_XDECREF(d);
    return ok;
}
static int to_ptr(PyObject *t, void **p) {
    PyObject *v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!v) return 0;
    *p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
static int to_int(PyObject *v, const char *name, int *out) {
    const long x = PyLong_AsLong(v);
    if (x == -1 && PyErr_Occurred()) return 0;
    if (x < INT_MIN || x > INT_MAX) {
        PyErr_Format(PyExc_OverflowError, "%s does not fit 32 bits", name);
        return 0;
    }
    *out = (int)x;
    return 1;
}
/* A tuple of n integers, by an attribute or a method without arguments. */
static int numbers(PyObject *v, int n, int64_t *out) {
    int ok = v && PyTuple_Check(v) && PyTuple_GET_SIZE(v) == n;
    for (int i = 0; ok && i < n; ++i) {
        out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
        ok = !(out[i] == -1 && PyErr_Occurred());
    }
    Py_XDECREF(v);
    return ok;
}
static int dims(PyObject *t, const char *name, int n, int64_t *d) {
    if (numbers(PyObject_GetAttr(t, s_shape), n, d)) return 1;
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s must have %d dimensions", name, n);
    return 0;
}
/* A T x H x D tensor with contiguous heads, of type `want` unless that is null. */
static int rows(PyObject *t, const char *name, int64_t T, int64_t H, int64_t D, PyObject *want, Rows *r) {
    int64_t d[3], s[3];
    if (!on_device(t, name) || (want && !same_type(t, name, want)) || !dims(t, name, 3, d)) return 0;
    if (d[0] != T || d[1] != H || d[2] != D) {
        PyErr_Format(PyExc_ValueError, "%s must be %lld x %lld x %lld, got %lld x %lld x %lld", name, (long long)T,
                     (long long)H, (long long)D, (long long)d[0], (long long)d[1], (long long)d[2]);
        return 0;
    }
    if (!numbers(PyObject_CallMethodNoArgs(t, s_stride), 3, s)) return 0;
    if (s[2] != 1 && D > 1) {
        PyErr_Format(PyExc_ValueError, "the last dimension of %s must be contiguous", name);
        return 0;
    }
    r->token = s[0];
    r->head = s[1];
    return to_ptr(t, &r->p);
}
/* A contiguous tensor of n values of type `want`. */
static int vector(PyObject *t, const char *name, int64_t n, PyObject *want, void **p) {
    if (!on_device(t, name) || !same_type(t, name, want)) return 0;
    PyObject *c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!c) return 0;
    Py_DECREF(c);
    if (c != Py_True) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
        return 0;
    }
    PyObject *m = PyObject_CallMethodNoArgs(t, s_numel);
    if (!m) return 0;
    const long long has = PyLong_AsLongLong(m);
    Py_DECREF(m);
    if (has != n) {
        if (!PyErr_Occurred())
            PyErr_Format(PyExc_ValueError, "%s has %lld elements, expected %lld", name, has, (long long)n);
        return 0;
    }
    return to_ptr(t, p);
}
static const int float_codes[3] = {PVMVMD_BF16, PVMVMD_F16, PVMVMD_F32};
/* The code of a tensor's type, and one of the dtype objects above. */
static int type_code(PyObject *t, const char *name, int field, int *code, PyObject **type) {
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return 0;
    *type = NULL;
    for (int i = 0; i < 3; ++i)
        if (d == t_float[i]) *type = t_float[i], *code = float_codes[i];
    if (field && d != Py_None && (d == t_int32 || d == t_uint32))
        *type = d == t_int32 ? t_int32 : t_uint32, *code = PVMVMD_FIELD;
    if (!*type) PyErr_Format(PyExc_TypeError, "%s must be a floating%s tensor, got %S", name, field ? " or field" : "", d);
    Py_DECREF(d);
    return *type != NULL;
}
static PyObject *pool_type(const pvmvmd_kv_pool *pool) {
    for (int i = 0; i < 2; ++i)
        if (pool->type == float_codes[i]) return t_float[i];
    return t_float[2]; /* which the library refuses */
}

/* The caller's stream: an integer, an object with cuda_stream, or None for the current one. */
static int stream_of(PyObject *s, void **out) {
    PyObject *v;
    if (s == Py_None) {
        PyObject *d = f_device == Py_None ? NULL : PyObject_CallNoArgs(f_device);
        if (f_device != Py_None && !d) return 0;
        v = d ? PyObject_CallOneArg(f_stream, d) : PyObject_CallNoArgs(f_stream);
        Py_XDECREF(d);
    } else {
        v = PyLong_Check(s) ? Py_NewRef(s) : PyObject_GetAttr(s, s_cuda_stream);
    }
    if (!v) return 0;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
static int address(PyObject *v, void **out) {
    *out = PyLong_AsVoidPtr(v);
    return !PyErr_Occurred();
}
static int arity(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    return n == want;
}
static int ready(Py_ssize_t n, Py_ssize_t want) {
    if (!f_rope) PyErr_SetString(PyExc_RuntimeError, "the library has not been opened");
    return f_rope && arity(n, want);
}
#define CALL(status, call)       \
    Py_BEGIN_ALLOW_THREADS       \
    status = call;               \
    Py_END_ALLOW_THREADS

/* rope(view, positions, x, out, scale, stream) */
static PyObject *rope(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    void *view, *pos, *stream;
    int64_t d[3];
    Rows x, out;
    PyObject *type;
    int in_code, out_code, status;
    if (!ready(n, 6) || !address(a[0], &view) || !dims(a[2], "x", 3, d) || !rows(a[2], "x", d[0], d[1], d[2], NULL, &x) ||
        !type_code(a[2], "x", 1, &in_code, &type) || !rows(a[3], "out", d[0], d[1], d[2], NULL, &out) ||
        !type_code(a[3], "out", 0, &out_code, &type) || !vector(a[1], "positions", d[0], t_int32, &pos))
        return NULL;
    const double scale = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred() || !stream_of(a[5], &stream)) return NULL;
    if (d[0] > INT_MAX || d[1] > INT_MAX || d[2] > INT_MAX) return PyLong_FromLong(PVMVMD_E_SHAPE);
    CALL(status, f_rope(view, pos, (int)d[0], (int)d[1], (int)d[2], x.p, in_code, x.token, x.head, (float)scale, out.p,
                        out_code, out.token, out.head, stream))
    return PyLong_FromLong(status);
}

/* append(pool, batch, view or 0, positions or None, scale, k, v, q or None, q_out, stream) */
static PyObject *append(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    void *view, *pos = NULL, *stream, *pp, *bp;
    int64_t d[3], dq[3] = {0, 0, 0};
    Rows k, v, q = {0}, out = {0};
    PyObject *type;
    int code, status;
    if (!ready(n, 10) || !address(a[0], &pp) || !address(a[1], &bp) || !address(a[2], &view)) return NULL;
    const pvmvmd_kv_pool *pool = pp;
    pvmvmd_kv_batch batch = *(const pvmvmd_kv_batch *)bp; /* (other threads' calls may use it with rows of theirs) */
    if (!dims(a[5], "k", 3, d) || !rows(a[5], "k", d[0], pool->heads, pool->dim, NULL, &k) ||
        !type_code(a[5], "k", 1, &code, &type) || !rows(a[6], "v", d[0], pool->heads, pool->dim, type, &v))
        return NULL;
    if (a[7] != Py_None &&
        (!dims(a[7], "q", 3, dq) || !rows(a[7], "q", d[0], dq[1], pool->dim, type, &q) ||
         !rows(a[8], "q_out", d[0], dq[1], pool->dim, pool_type(pool), &out)))
        return NULL;
    if (a[3] != Py_None && !vector(a[3], "positions", d[0], t_int32, &pos)) return NULL;
    const double scale = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred() || !stream_of(a[9], &stream)) return NULL;
    if (d[0] > INT_MAX || dq[1] > INT_MAX) return PyLong_FromLong(PVMVMD_E_SHAPE);
    batch.T = (int)d[0];
    CALL(status, f_append(pool, &batch, view, pos, code, (float)scale, k.p, k.token, k.head, v.p, v.token, v.head,
                          (int)dq[1], q.p, q.token, q.head, out.p, out.token, out.head, stream))
    return PyLong_FromLong(status);
}

/* attend(pool, batch, q, out, lse or None, scale or None, causal, window, accumulate, stream) */
static PyObject *attend(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    void *pp, *bp, *lse = NULL, *stream;
    int64_t d[3];
    Rows q, out;
    int window, status;
    if (!ready(n, 10) || !address(a[0], &pp) || !address(a[1], &bp)) return NULL;
    const pvmvmd_kv_pool *pool = pp;
    pvmvmd_kv_batch batch = *(const pvmvmd_kv_batch *)bp; /* (other threads' calls may use it with rows of theirs) */
    if (!dims(a[2], "q", 3, d) || !rows(a[2], "q", d[0], d[1], pool->dim, pool_type(pool), &q) ||
        !rows(a[3], "out", d[0], d[1], pool->dim, pool_type(pool), &out) ||
        (a[4] != Py_None && !vector(a[4], "lse", d[0] * d[1], t_float[2], &lse)))
        return NULL;
    const double scale = a[5] == Py_None ? pow((double)pool->dim, -0.5) : PyFloat_AsDouble(a[5]);
    const int causal = PyObject_IsTrue(a[6]), accumulate = PyObject_IsTrue(a[8]);
    if (PyErr_Occurred() || !to_int(a[7], "window", &window) || !stream_of(a[9], &stream)) return NULL;
    if (d[0] > INT_MAX || d[1] > INT_MAX) return PyLong_FromLong(PVMVMD_E_SHAPE);
    batch.T = (int)d[0];
    CALL(status, f_attend(pool, &batch, (int)d[1], q.p, q.token, q.head, (float)scale, causal, window, accumulate, out.p,
                          out.token, out.head, lse, stream))
    return PyLong_FromLong(status);
}

/* evict(pool, batch, budget, recent, new_table, new_lens, stream) */
static PyObject *evict(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    void *pp, *bp, *table, *lens, *stream;
    int64_t d[2], s[2];
    int budget, recent, status;
    if (!ready(n, 7) || !address(a[0], &pp) || !address(a[1], &bp)) return NULL;
    const pvmvmd_kv_batch *batch = bp;
    if (!to_int(a[2], "budget", &budget) || !to_int(a[3], "recent", &recent)) return NULL;
    if (!on_device(a[4], "new_table") || !same_type(a[4], "new_table", t_int32) || !dims(a[4], "new_table", 2, d) ||
        !numbers(PyObject_CallMethodNoArgs(a[4], s_stride), 2, s) || d[0] != batch->B || (d[1] > 1 && s[1] != 1) ||
        d[1] > INT_MAX) {
        PyErr_SetString(PyExc_ValueError, "new_table must be an int32 CUDA tensor B x pages with contiguous rows");
        return NULL;
    }
    if (!to_ptr(a[4], &table) || !vector(a[5], "new_lens", batch->B, t_int32, &lens) || !stream_of(a[6], &stream))
        return NULL;
    CALL(status, f_evict(pp, batch, budget, recent, table, s[0], (int)d[1], lens, stream))
    return PyLong_FromLong(status);
}

/* open(library handle, bfloat16, float16, float32, int32, uint32 or None, stream, device or None) */
static PyObject *open_library(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    void *h;
    if (!arity(n, 8) || !address(a[0], &h)) return NULL;
    f_rope = (__typeof__(f_rope))dlsym(h, "pvmvmd_rope");
    f_append = (__typeof__(f_append))dlsym(h, "pvmvmd_kv_append");
    f_attend = (__typeof__(f_attend))dlsym(h, "pvmvmd_paged_attention");
    f_evict = (__typeof__(f_evict))dlsym(h, "pvmvmd_kv_evict");
    if (!f_rope || !f_append || !f_attend || !f_evict) {
        PyErr_SetString(PyExc_ImportError, "libpvmvmd.so does not have the calls of the client's attention");
        return NULL;
    }
    PyObject **to[7] = {&t_float[0], &t_float[1], &t_float[2], &t_int32, &t_uint32, &f_stream, &f_device};
    for (int i = 0; i < 7; ++i) Py_XSETREF(*to[i], Py_NewRef(a[1 + i]));
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"open", (PyCFunction)(void (*)(void))open_library, METH_FASTCALL, NULL},
                                {"rope", (PyCFunction)(void (*)(void))rope, METH_FASTCALL, NULL},
                                {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, NULL},
                                {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, NULL},
                                {"evict", (PyCFunction)(void (*)(void))evict, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    static const char *const names[8] = {"is_cuda", "dtype", "shape",         "stride",
                                         "data_ptr", "numel", "is_contiguous", "cuda_stream"};
    PyObject **const to[8] = {&s_is_cuda,  &s_dtype, &s_shape,         &s_stride,
                              &s_data_ptr, &s_numel, &s_is_contiguous, &s_cuda_stream};
    for (int i = 0; i < 8; ++i)
        if (!(*to[i] = PyUnicode_InternFromString(names[i]))) return NULL;
    return PyModule_Create(&module);
}
