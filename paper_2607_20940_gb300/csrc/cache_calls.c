/* Arguments of the 4-bit cache's per-token calls, taken from torch tensors in C.
 *
 * An append or an attention of a few tokens is some microseconds of device time, and
 * reading shapes, strides and pointers from Python and through ctypes takes 2 to 3 of
 * them a call. Each function here makes the call where its arguments are what nearly every
 * call has, and returns None, without having called, where they are not: msf.py then looks
 * at them one by one and raises what is wrong. Nothing is kept from one call to the next. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>
#include <string.h>

#include "../../include/msf_cache.h"

static PyObject *s_dtype, *s_is_cuda, *s_shape, *s_stride, *s_data_ptr;
static PyObject *bfloat16, *float32, *int32;

typedef struct {
    void* p;
    long long shape[4], stride[4];
} rows_t;

static int longs(PyObject* tuple, int n, long long* out) {
    if (!tuple || !PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != n) return 0;
    for (int i = 0; i < n; ++i) {
        out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
        if (out[i] == -1 && PyErr_Occurred()) return 0;
    }
    return 1;
}

static int attr_is(PyObject* t, PyObject* name, PyObject* want) {
    PyObject* x = PyObject_GetAttr(t, name);
    const int same = x == want;
    Py_XDECREF(x);
    return same;
}

/* A device tensor of this type with n dimensions. */
static int look(PyObject* t, PyObject* dtype, int n, rows_t* r) {
    if (!attr_is(t, s_dtype, dtype) || !attr_is(t, s_is_cuda, Py_True)) return 0;
    PyObject* x = PyObject_GetAttr(t, s_shape);
    int fine = longs(x, n, r->shape);
    Py_XDECREF(x);
    if (!fine) return 0;
    x = PyObject_CallMethodNoArgs(t, s_stride);
    fine = longs(x, n, r->stride);
    Py_XDECREF(x);
    if (!fine) return 0;
    x = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!x) return 0;
    r->p = PyLong_AsVoidPtr(x);
    Py_DECREF(x);
    return !PyErr_Occurred();
}

/* A list of n entries, or None. */
static int look_list(PyObject* t, long long n, const int32_t** p) {
    rows_t r;
    *p = NULL;
    if (t == Py_None) return 1;
    if (!look(t, int32, 1, &r) || r.shape[0] != n || (n > 1 && r.stride[0] != 1)) return 0;
    *p = (const int32_t*)r.p;
    return 1;
}

/* Rows of heads whose strides the library takes as they are. */
static int look_rows(PyObject* t, rows_t* r) {
    return look(t, bfloat16, 4, r) && r->stride[3] == 1 && !((r->stride[0] | r->stride[1] | r->stride[2]) & 7);
}

static PyObject* not_here(void) {
    PyErr_Clear();
    Py_RETURN_NONE;
}

typedef msf_status (*rows_fn)(msf_cache_t, int32_t, const int32_t*, const int32_t*, int32_t, int32_t, void*, void*,
                              const int64_t*, void*);
typedef msf_status (*attend_fn)(msf_cache_t, int32_t, const int32_t*, int32_t, const msf_cache_attention*, void*);

static int fits(long long x) { return x >= 0 && x <= INT32_MAX; }

/* rows(fn, cache, layer, k, v, seqs, at, kv_heads, head_dim, stream): msf_cache_write or msf_cache_read. */
static PyObject* rows(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 10) return not_here();
    rows_t k, v;
    const int32_t *seqs, *at;
    const rows_fn fn = (rows_fn)(uintptr_t)PyLong_AsVoidPtr(a[0]);
    const msf_cache_t cache = (msf_cache_t)PyLong_AsVoidPtr(a[1]);
    const long long layer = PyLong_AsLongLong(a[2]), kv_heads = PyLong_AsLongLong(a[7]), head_dim = PyLong_AsLongLong(a[8]);
    void* const stream = PyLong_AsVoidPtr(a[9]);
    if (PyErr_Occurred() || !fn || !look_rows(a[3], &k) || !look_rows(a[4], &v)) return not_here();
    if (memcmp(k.shape, v.shape, sizeof k.shape) || memcmp(k.stride, v.stride, sizeof k.stride)) return not_here();
    if (k.shape[2] != kv_heads || k.shape[3] != head_dim || !fits(layer) || !fits(k.shape[0]) || !fits(k.shape[1])) return not_here();
    if (!look_list(a[5], k.shape[0], &seqs) || !look_list(a[6], k.shape[0], &at)) return not_here();
    const int64_t strides[3] = {k.stride[0], k.stride[1], k.stride[2]};
    msf_status status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(cache, (int32_t)layer, seqs, at, (int32_t)k.shape[0], (int32_t)k.shape[1], k.p, v.p, strides, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* attend(fn, cache, layer, q, out, lse, base_out, base_lse, seqs, causal, scale, skip, head_dim, stream). */
static PyObject* attend(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 14) return not_here();
    rows_t q, out, base, lse, base_lse;
    const int32_t* seqs;
    const attend_fn fn = (attend_fn)(uintptr_t)PyLong_AsVoidPtr(a[0]);
    const msf_cache_t cache = (msf_cache_t)PyLong_AsVoidPtr(a[1]);
    const long long layer = PyLong_AsLongLong(a[2]), skip = PyLong_AsLongLong(a[11]), head_dim = PyLong_AsLongLong(a[12]);
    const double scale = PyFloat_AsDouble(a[10]);
    const int causal = PyObject_IsTrue(a[9]);
    void* const stream = PyLong_AsVoidPtr(a[13]);
    if (PyErr_Occurred() || !fn || !look_rows(a[3], &q) || !look_rows(a[4], &out)) return not_here();
    if (memcmp(q.shape, out.shape, sizeof q.shape) || q.shape[3] != head_dim) return not_here();
    if (!fits(layer) || !fits(skip) || !fits(q.shape[0]) || !fits(q.shape[1]) || !fits(q.shape[2])) return not_here();
    const int has_lse = a[5] != Py_None, has_base = a[6] != Py_None, has_base_lse = a[7] != Py_None;
    if (has_base && a[6] != a[4]) {
        if (!look_rows(a[6], &base) || memcmp(base.shape, out.shape, sizeof out.shape) || memcmp(base.stride, out.stride, sizeof out.stride))
            return not_here();
    } else {
        base.p = has_base ? out.p : NULL;
    }
    const long long want[3] = {q.shape[0], q.shape[2], q.shape[1]};
    if (has_lse && (!look(a[5], float32, 3, &lse) || memcmp(lse.shape, want, sizeof want) || (lse.stride[2] != 1 && want[2] > 1)))
        return not_here();
    if (has_base_lse && (a[7] != a[5] || !has_lse)) {
        if (!look(a[7], float32, 3, &base_lse) || memcmp(base_lse.shape, want, sizeof want) || (base_lse.stride[2] != 1 && want[2] > 1))
            return not_here();
        if (has_lse && memcmp(base_lse.stride, lse.stride, 2 * sizeof lse.stride[0])) return not_here();
    } else if (has_base_lse) {
        base_lse = lse;
    }
    if (!look_list(a[8], q.shape[0], &seqs)) return not_here();
    msf_cache_attention x;
    memset(&x, 0, sizeof x);
    x.q = q.p;
    x.out = out.p;
    x.base_out = base.p;
    x.lse = has_lse ? (float*)lse.p : NULL;
    x.base_lse = has_base_lse ? (const float*)base_lse.p : NULL;
    for (int i = 0; i < 3; ++i) {
        x.q_strides[i] = q.stride[i];
        x.out_strides[i] = out.stride[i];
    }
    for (int i = 0; i < 2; ++i) x.lse_strides[i] = has_lse ? lse.stride[i] : has_base_lse ? base_lse.stride[i] : 0;
    x.queries = (int32_t)q.shape[1];
    x.heads = (int32_t)q.shape[2];
    x.causal = causal;
    x.skip = (int32_t)skip;
    x.softmax_scale = (float)scale;
    msf_status status;
    Py_BEGIN_ALLOW_THREADS
    status = fn(cache, (int32_t)layer, seqs, (int32_t)q.shape[0], &x, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* types(bfloat16, float32, int32): torch's types, once. */
static PyObject* types(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 3) {
        PyErr_SetString(PyExc_TypeError, "types(bfloat16, float32, int32)");
        return NULL;
    }
    PyObject** const to[3] = {&bfloat16, &float32, &int32};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[i]);
        Py_XSETREF(*to[i], a[i]);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"rows", (PyCFunction)(void (*)(void))rows, METH_FASTCALL, "msf_cache_write or msf_cache_read: a status, or None"},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, "msf_cache_attend: a status, or None"},
    {"types", (PyCFunction)(void (*)(void))types, METH_FASTCALL, "torch's types"},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cache_calls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__cache_calls(void) {
    s_dtype = PyUnicode_InternFromString("dtype");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    if (!s_dtype || !s_is_cuda || !s_shape || !s_stride || !s_data_ptr) return NULL;
    return PyModule_Create(&module);
}
