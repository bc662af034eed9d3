/* _decode.c — argument marshalling of the decode operators (decode.py) for
 * CPython. A decode step makes these calls every few microseconds; from ctypes
 * a call with its checks costs more than its kernel. The checks are the ones
 * that the C ABI cannot make: a tensor's type, size, strides and device.
 *
 * Tensors are asked through their Python attributes (no torch headers); the
 * library's functions are called through the addresses that setup() is given.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "vbq.h"

static __typeof__(&vbq_kv_append) p_append;
static __typeof__(&vbq_kv_read) p_read;
static __typeof__(&vbq_kv_attend) p_attend;
static __typeof__(&vbq_residual_norm) p_norm;
static __typeof__(&vbq_sample) p_sample;

static PyObject *dt_f32, *dt_bf16, *dt_i16, *dt_i32, *raw_stream, *current_device;
static PyObject *s_dtype, *s_shape, *s_stride, *s_numel, *s_contiguous, *s_device, *s_ptr, *s_nbytes, *s_cuda_stream;

enum { F32 = 1, BF16 = 2, I32 = 4 };            /* BF16: or its bit patterns in int16 */

/* ---- asking a tensor; every function returns -1 with an exception set on failure ---- */

static int long_of(PyObject* o, long long* v) { /* takes o */
    if (!o) return -1;
    *v = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return *v == -1 && PyErr_Occurred() ? -1 : 0;
}

static int ask(PyObject* t, PyObject* method, long long* v) { return long_of(PyObject_CallMethodNoArgs(t, method), v); }

static int kind_of(PyObject* t) {               /* 0: another type */
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    const int k = d == dt_f32 ? F32 : d == dt_bf16 || d == dt_i16 ? BF16 : d == dt_i32 ? I32 : 0;
    Py_DECREF(d);
    return k;
}

/* The GPU of a call's first tensor. The library launches on the current device, whatever the addresses that it is given. */
static int device_of(PyObject* t, long long* dev) {
    long long current;
    if (ask(t, s_device, dev) < 0) return -1;
    if (*dev < 0) {
        PyErr_SetString(PyExc_ValueError, "tensors must be on a GPU");
        return -1;
    }
    if (current_device == Py_None) return 0;    /* a process with one GPU */
    if (long_of(PyObject_CallNoArgs(current_device), &current) < 0) return -1;
    if (*dev != current) {
        PyErr_Format(PyExc_ValueError, "tensors are on cuda:%lld, but the current device is cuda:%lld", *dev, current);
        return -1;
    }
    return 0;
}

#define DIMS 8

/* Up to DIMS numbers of a tuple; their count. */
static int tuple_of(PyObject* o, long long* v) { /* takes o */
    if (!o) return -1;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) > DIMS) {
        Py_DECREF(o);
        PyErr_SetString(PyExc_ValueError, "expected a tensor of at most 8 dimensions");
        return -1;
    }
    const int n = (int)PyTuple_GET_SIZE(o);
    for (int i = 0; i < n; ++i) v[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(o, i));
    Py_DECREF(o);
    return PyErr_Occurred() ? -1 : n;
}
static int shape_of(PyObject* t, long long* v) { return tuple_of(PyObject_GetAttr(t, s_shape), v); }
static int strides_of(PyObject* t, long long* v) { return tuple_of(PyObject_CallMethodNoArgs(t, s_stride), v); }

static int contiguous(PyObject* t) {
    PyObject* o = PyObject_CallMethodNoArgs(t, s_contiguous);
    if (!o) return -1;
    const int yes = o == Py_True;
    Py_DECREF(o);
    return yes;
}

/* Address of a contiguous tensor of n elements of one of the kinds on the device. */
static int dense(PyObject* t, int kinds, long long n, long long dev, const char* name, void** p) {
    long long m, d, a;
    const int k = kind_of(t);
    if (k < 0 || ask(t, s_numel, &m) < 0 || ask(t, s_device, &d) < 0) return -1;
    const int c = contiguous(t);
    if (c < 0) return -1;
    if (!(k & kinds) || m != n || d != dev || !c) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s tensor of %lld elements on cuda:%lld, got %lld on device %lld%s%s", name,
                     kinds == F32 ? "float32" : kinds == BF16 ? "bfloat16" : kinds == I32 ? "int32" : "float32 or bfloat16", n, dev, m, d,
                     c ? "" : ", not contiguous", k & kinds ? "" : ", of another type");
        return -1;
    }
    if (ask(t, s_ptr, &a) < 0) return -1;
    *p = (void*)(intptr_t)a;
    return 0;
}

/* VBQ_F32 or VBQ_BF16. */
static int type_of(PyObject* t) {
    const int k = kind_of(t);
    if (k < 0) return -1;
    if (k == F32) return VBQ_F32;
    if (k == BF16) return VBQ_BF16;
    PyErr_SetString(PyExc_ValueError, "expected a float32 or bfloat16 tensor");
    return -1;
}

static int stream_of(PyObject* s, long long dev, void** out) {
    long long v;
    if (s == Py_None) {
        PyObject* d = PyLong_FromLongLong(dev);
        if (!d) return -1;
        PyObject* r = PyObject_CallOneArg(raw_stream, d);
        Py_DECREF(d);
        if (long_of(r, &v) < 0) return -1;
    } else if (PyLong_Check(s)) {
        v = PyLong_AsLongLong(s);
        if (v == -1 && PyErr_Occurred()) return -1;
    } else if (long_of(PyObject_GetAttr(s, s_cuda_stream), &v) < 0) {
        return -1;
    }
    *out = (void*)(intptr_t)v;
    return 0;
}

/* Two arguments that a call takes together or not at all. */
static int together(PyObject* a, PyObject* b, const char* names) {
    if ((a == Py_None) == (b == Py_None)) return 0;
    PyErr_Format(PyExc_ValueError, "%s go together", names);
    return -1;
}

/* ---- a cache call's table and rows ---- */

typedef struct {
    const vbq_kv_cache* cache;
    long long dev;
    const int32_t *table, *pos;
    long long stride, pages, batch, rows;
} Rows;

static int rows_of(PyObject* cache, PyObject* cache_dev, PyObject* table, PyObject* pos, Rows* r) {
    long long v[DIMS], s[DIMS], a, d;
    const int kt = kind_of(table);
    if (kt < 0) return -1;
    int n = shape_of(table, v);
    if (n < 0 || strides_of(table, s) < 0) return -1;
    if (kt != I32 || n != 2 || (s[1] != 1 && v[1] > 1)) {
        PyErr_SetString(PyExc_ValueError, "table must be an int32 tensor (batch, pages) with dense rows");
        return -1;
    }
    r->stride = s[0];
    r->pages = v[1];
    r->batch = v[0];
    const int kp = kind_of(pos);
    if (kp < 0) return -1;
    n = shape_of(pos, v);
    if (n < 0) return -1;
    const int c = contiguous(pos);
    if (c < 0) return -1;
    if (kp != I32 || n != 2 || !c || v[0] != r->batch) {
        PyErr_SetString(PyExc_ValueError, "pos must be a contiguous int32 tensor (batch, rows)");
        return -1;
    }
    r->rows = v[1];
    if (device_of(table, &r->dev) < 0 || ask(pos, s_device, &d) < 0) return -1;
    const long long cd = PyLong_AsLongLong(cache_dev);
    if (cd == -1 && PyErr_Occurred()) return -1;
    if (d != r->dev || cd != r->dev) {
        PyErr_SetString(PyExc_ValueError, "table, pos and the cache must be on one GPU");
        return -1;
    }
    if (r->pages > INT32_MAX || r->batch > INT32_MAX || r->rows > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "table or pos is too large");
        return -1;
    }
    a = PyLong_AsLongLong(cache);
    if (a == -1 && PyErr_Occurred()) return -1;
    r->cache = (const vbq_kv_cache*)(intptr_t)a;
    if (ask(table, s_ptr, &a) < 0) return -1;
    r->table = (const int32_t*)(intptr_t)a;
    if (ask(pos, s_ptr, &a) < 0) return -1;
    r->pos = (const int32_t*)(intptr_t)a;
    return 0;
}

/* A (batch, rows, heads, head_dim) tensor whose rows are dense and evenly spaced: its address and the elements between rows. */
static int rows_tensor(PyObject* t, const Rows* r, long long heads, const char* name, void** p, long long* stride) {
    long long v[DIMS], s[DIMS], d, a;
    const int n = shape_of(t, v);
    if (n < 0 || strides_of(t, s) < 0 || ask(t, s_device, &d) < 0) return -1;
    const long long hd = r->cache->head_dim;
    if (n != 4 || v[0] != r->batch || v[1] != r->rows || v[2] != heads || v[3] != hd || d != r->dev) {
        PyErr_Format(PyExc_ValueError, "%s must have shape (%lld, %lld, %lld, %lld) on cuda:%lld", name, r->batch, r->rows, heads, hd, r->dev);
        return -1;
    }
    if (s[3] != 1 || (heads > 1 && s[2] != hd) || (r->rows > 1 && r->batch > 1 && s[0] != r->rows * s[1])) {
        PyErr_Format(PyExc_ValueError, "%s's rows must be dense and evenly spaced", name);
        return -1;
    }
    *stride = r->rows > 1 ? s[1] : s[0];
    if (ask(t, s_ptr, &a) < 0) return -1;
    *p = (void*)(intptr_t)a;
    return 0;
}

#define NEED(count)                                                                                     \
    do {                                                                                                \
        if (n != (count)) {                                                                             \
            PyErr_Format(PyExc_TypeError, "%s takes %d arguments, got %zd", __func__, (int)(count), n); \
            return NULL;                                                                                \
        }                                                                                               \
    } while (0)

/* append(cache address, cache device, table, pos, k, v, q, cos, sin, q_out, stream) */
static PyObject* append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(11);
    Rows r;
    void *k, *v, *q = NULL, *q_out = NULL, *cos = NULL, *sin = NULL, *st;
    long long ks, vs, qs = 0, heads = 0, rot = 0, rot_rows = 0, shape[DIMS];
    if (rows_of(a[0], a[1], a[2], a[3], &r) < 0 || together(a[6], a[9], "q and q_out") < 0 || together(a[7], a[8], "cos and sin") < 0) return NULL;
    const int type = type_of(a[4]), tv = type_of(a[5]);
    if (type < 0 || tv < 0) return NULL;
    int tq = type;
    if (a[6] != Py_None && (tq = type_of(a[6])) < 0) return NULL;
    if (tv != type || tq != type) {
        PyErr_SetString(PyExc_ValueError, "q, k and v must have one type");
        return NULL;
    }
    if (rows_tensor(a[4], &r, r.cache->kv_heads, "k", &k, &ks) < 0 || rows_tensor(a[5], &r, r.cache->kv_heads, "v", &v, &vs) < 0) return NULL;
    if (a[6] != Py_None) {
        const int m = shape_of(a[6], shape);
        if (m < 0) return NULL;
        heads = m == 4 ? shape[2] : -1;
        if (heads < 0 || heads > (1 << 20)) {
            PyErr_SetString(PyExc_ValueError, "q must have shape (batch, rows, heads, head_dim)");
            return NULL;
        }
        if (rows_tensor(a[6], &r, heads, "q", &q, &qs) < 0 ||
            dense(a[9], BF16, r.batch * r.rows * heads * r.cache->head_dim, r.dev, "q_out", &q_out) < 0)
            return NULL;
    }
    if (a[7] != Py_None) {
        const int m = shape_of(a[7], shape);
        if (m < 0) return NULL;
        if (m != 2 || shape[1] > (1 << 20)) {
            PyErr_SetString(PyExc_ValueError, "cos must have shape (positions, rot_dim / 2)");
            return NULL;
        }
        rot_rows = shape[0];
        rot = 2 * shape[1];
        if (dense(a[7], F32, rot_rows * shape[1], r.dev, "cos", &cos) < 0 || dense(a[8], F32, rot_rows * shape[1], r.dev, "sin", &sin) < 0)
            return NULL;
    }
    if (stream_of(a[10], r.dev, &st) < 0) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = p_append(r.cache, r.table, r.stride, (int)r.pages, r.pos, (int)r.batch, (int)r.rows, q, qs, (int)heads, k, ks, v, vs, type, cos,
                      sin, (int)rot, rot_rows, q_out, st);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

/* read(cache address, cache device, table, pos, k_out or False, v_out or False, stream) */
static PyObject* read_(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(7);
    Rows r;
    void *k = NULL, *v = NULL, *st;
    if (rows_of(a[0], a[1], a[2], a[3], &r) < 0) return NULL;
    const long long m = r.batch * r.rows * r.cache->kv_heads * r.cache->head_dim;
    if (a[4] != Py_False && dense(a[4], F32, m, r.dev, "k_out", &k) < 0) return NULL;
    if (a[5] != Py_False && dense(a[5], F32, m, r.dev, "v_out", &v) < 0) return NULL;
    if (stream_of(a[6], r.dev, &st) < 0) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = p_read(r.cache, r.table, r.stride, (int)r.pages, r.pos, (int)r.batch, (int)r.rows, k, v, st);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

/* attend(cache address, cache device, table, pos, q, scale or None, window, out, workspace, stream) */
static PyObject* attend(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(10);
    Rows r;
    void *q, *out, *st;
    long long shape[DIMS], ws, bytes, d;
    if (rows_of(a[0], a[1], a[2], a[3], &r) < 0) return NULL;
    const int m = shape_of(a[4], shape);
    if (m < 0) return NULL;
    if (m != 4 || shape[0] != r.batch || shape[1] != r.rows || shape[3] != r.cache->head_dim || shape[2] > (1 << 20)) {
        PyErr_Format(PyExc_ValueError, "q must have shape (%lld, %lld, heads, %d)", r.batch, r.rows, r.cache->head_dim);
        return NULL;
    }
    const long long count = shape[0] * shape[1] * shape[2] * shape[3];
    double scale;
    if (a[5] == Py_None) {
        const int hd = r.cache->head_dim;       /* 64, 128 or 256: the exact power or its nearest */
        scale = hd == 64 ? 0.125 : hd == 256 ? 0.0625 : 0.08838834764831845;
    } else {
        scale = PyFloat_AsDouble(a[5]);
        if (scale == -1.0 && PyErr_Occurred()) return NULL;
    }
    const long window = PyLong_AsLong(a[6]);
    if (window == -1 && PyErr_Occurred()) return NULL;
    if (window > INT32_MAX || window < INT32_MIN) {
        PyErr_SetString(PyExc_ValueError, "window is out of range");
        return NULL;
    }
    if (dense(a[4], BF16, count, r.dev, "q", &q) < 0 || dense(a[7], BF16, count, r.dev, "out", &out) < 0) return NULL;
    const int c = contiguous(a[8]);
    if (c < 0 || ask(a[8], s_device, &d) < 0 || ask(a[8], s_ptr, &ws) < 0 || long_of(PyObject_GetAttr(a[8], s_nbytes), &bytes) < 0) return NULL;
    if (!c || d != r.dev) {
        PyErr_SetString(PyExc_ValueError, "workspace must be a contiguous tensor on the cache's GPU");
        return NULL;
    }
    if (stream_of(a[9], r.dev, &st) < 0) return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = p_attend(r.cache, r.table, r.stride, (int)r.pages, r.pos, (int)r.batch, (int)r.rows, q, (int)shape[2], (float)scale, (int)window,
                      out, (void*)(intptr_t)ws, (size_t)bytes, st);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

/* norm(x, residual, weight, eps, out, residual_out, stream) */
static PyObject* norm(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(7);
    long long dev, count, shape[DIMS], width;
    void *x, *w, *out, *r = NULL, *ro = NULL, *st;
    if (device_of(a[0], &dev) < 0 || ask(a[0], s_numel, &count) < 0 || together(a[1], a[5], "residual and residual_out") < 0) return NULL;
    const int xt = type_of(a[0]), m = xt < 0 ? -1 : shape_of(a[0], shape);
    if (m < 0) return NULL;
    if (m == 0) {
        PyErr_SetString(PyExc_ValueError, "x must have a dimension to normalise");
        return NULL;
    }
    width = shape[m - 1];
    int rt = VBQ_BF16;
    if (a[1] != Py_None) {
        if ((rt = type_of(a[1])) < 0) return NULL;
        const int k = rt == VBQ_F32 ? F32 : BF16;
        if (dense(a[1], k, count, dev, "residual", &r) < 0) return NULL;
        if (a[5] == a[1])
            ro = r;
        else if (dense(a[5], k, count, dev, "residual_out", &ro) < 0)
            return NULL;
    }
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) return NULL;
    if (dense(a[0], xt == VBQ_F32 ? F32 : BF16, count, dev, "x", &x) < 0 || dense(a[2], F32, width, dev, "weight", &w) < 0 ||
        dense(a[4], BF16, count, dev, "out", &out) < 0 || stream_of(a[6], dev, &st) < 0)
        return NULL;
    if (width > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "x is too wide");
        return NULL;
    }
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = p_norm(x, xt, r, rt, w, (float)eps, width ? count / width : 0, (int)width, out, ro, st);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

/* sample(logits, temperature, top_k, top_p, min_p, u, tokens, probs or False, kept or False, stream) */
static PyObject* sample(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(10);
    long long dev, shape[DIMS], stride[DIMS], p;
    void *t, *k, *tp, *mp, *u, *tok, *pr = NULL, *ke = NULL, *st;
    if (device_of(a[0], &dev) < 0) return NULL;
    const int type = type_of(a[0]), m = type < 0 ? -1 : shape_of(a[0], shape);
    if (m < 0 || strides_of(a[0], stride) < 0) return NULL;
    if (m != 2 || (stride[1] != 1 && shape[1] > 1) || shape[0] > INT32_MAX || shape[1] > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "logits must have shape (batch, vocab) and dense rows");
        return NULL;
    }
    const long long b = shape[0];
    if (dense(a[1], F32, b, dev, "temperature", &t) < 0 || dense(a[2], I32, b, dev, "top_k", &k) < 0 ||
        dense(a[3], F32, b, dev, "top_p", &tp) < 0 || dense(a[4], F32, b, dev, "min_p", &mp) < 0 || dense(a[5], F32, b, dev, "u", &u) < 0 ||
        dense(a[6], I32, b, dev, "tokens", &tok) < 0 || (a[7] != Py_False && dense(a[7], F32, b, dev, "probs", &pr) < 0) ||
        (a[8] != Py_False && dense(a[8], I32, b, dev, "kept", &ke) < 0) || ask(a[0], s_ptr, &p) < 0 || stream_of(a[9], dev, &st) < 0)
        return NULL;
    int status;
    Py_BEGIN_ALLOW_THREADS;
    status = p_sample((const void*)(intptr_t)p, stride[0], type, (int)b, (int)shape[1], t, k, tp, mp, u, tok, pr, ke, st);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(status);
}

/* setup(float32, bfloat16, int16, int32, raw_stream, current_device or None, addresses of the five functions) */
static PyObject* setup(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    (void)self;
    NEED(11);
    long long f[5];
    for (int i = 0; i < 5; ++i) {
        f[i] = PyLong_AsLongLong(a[6 + i]);
        if (f[i] == -1 && PyErr_Occurred()) return NULL;
    }
    PyObject** keep[6] = {&dt_f32, &dt_bf16, &dt_i16, &dt_i32, &raw_stream, &current_device};
    for (int i = 0; i < 6; ++i) {
        Py_INCREF(a[i]);
        Py_XSETREF(*keep[i], a[i]);
    }
    p_append = (__typeof__(p_append))(intptr_t)f[0];
    p_read = (__typeof__(p_read))(intptr_t)f[1];
    p_attend = (__typeof__(p_attend))(intptr_t)f[2];
    p_norm = (__typeof__(p_norm))(intptr_t)f[3];
    p_sample = (__typeof__(p_sample))(intptr_t)f[4];
    Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))(f), METH_FASTCALL
static PyMethodDef methods[] = {
    {"setup", FAST(setup), NULL},   {"append", FAST(append), NULL}, {"read", FAST(read_), NULL}, {"attend", FAST(attend), NULL},
    {"norm", FAST(norm), NULL},     {"sample", FAST(sample), NULL}, {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_decode", "Marshalling of the decode operators' calls.", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__decode(void) {
    const struct { PyObject** to; const char* name; } names[] = {
        {&s_dtype, "dtype"},     {&s_shape, "shape"},     {&s_stride, "stride"}, {&s_numel, "numel"},       {&s_contiguous, "is_contiguous"},
        {&s_device, "get_device"}, {&s_ptr, "data_ptr"}, {&s_nbytes, "nbytes"}, {&s_cuda_stream, "cuda_stream"}};
    for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!(*names[i].to = PyUnicode_InternFromString(names[i].name))) return NULL;
    return PyModule_Create(&module);
}
