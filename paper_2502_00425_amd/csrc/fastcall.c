// The way from Python to a launch for the calls that decode and short prompts make by the dozen: what
// binding.py does for them in Python and ctypes, in C.  A call passes the same checks on the same methods
// of its tensors (shape, stride, data_ptr, is_contiguous), reads the stream through the same functions of
// torch and releases the interpreter lock while the library runs.  Anything out of the ordinary -- a
// method that raises an error, a number that is not a plain int or float, a layout the checks refuse --
// returns NotImplemented before the library is called, and binding.py goes its own way, which also
// words the errors.  Nothing is kept from one call for another.
//
// A call through this file costs the host 1.0 us beside the launch, through ctypes 3.3 (512 -> 512 at T = 64, a 3.8 us
// kernel: 6.0 -> 4.0, 6.4 -> 5.0 and 6.8 -> 4.9 us a call on three machines).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "mquant.h"

static PyObject *s_shape, *s_stride, *s_data_ptr, *s_is_contiguous, *s_dtype, *s_get_device;

// What setup() gives a module object: torch.cuda.is_initialized, the current device, its raw stream, and the library's
// entries.  Every load of the package has a module, and so a library, of its own.
typedef struct {
    PyObject *f_initialized, *f_device, *f_stream;
    int (*prefill)(const void *, int64_t, const int32_t *, const uint8_t *, const void *, void *, int64_t, int32_t, int32_t,
                   int32_t, int32_t, float, float, int32_t, void *, int64_t, mquant_stream_t);
    int (*prefill_static)(const void *, int64_t, const int32_t *, const uint8_t *, const void *, void *, int64_t, int32_t,
                          int32_t, int32_t, int32_t, float, float, int32_t, mquant_stream_t);
    int (*decode)(const void *, int64_t, const uint8_t *, const void *, void *, int64_t, int32_t, int32_t, int32_t, int32_t,
                  float, float, int32_t, mquant_stream_t);
    int (*decode_grouped)(const void *, int64_t, int32_t, int32_t, int32_t, float, float, int32_t, const mquant_linear_t *,
                          int32_t, mquant_stream_t);
    int (*gemv_grouped)(const int8_t *, int32_t, int32_t, int32_t, float, float, const mquant_linear_t *, int32_t,
                        mquant_stream_t);
    int (*quant)(const void *, int64_t, const int32_t *, int8_t *, int32_t, int32_t, int32_t, float, float, int32_t,
                 mquant_stream_t);
    int (*weight_only)(const void *, int64_t, const uint8_t *, void *, int64_t, int32_t, int32_t, int32_t, mquant_stream_t);
    // setup_serving(): torch.float16, torch.float32, torch.int32 and the entries of the serving step
    PyObject *f16, *f32, *i32;
    __typeof__(&mquant_qk_norm_rope) norm;
    __typeof__(&mquant_kv_append) append;
    __typeof__(&mquant_paged_attention) attention;
    __typeof__(&mquant_lora_apply) lora;
} State;

// ---- readers: 1 on success, 0 where the slow way has to look.  An interrupt, an exit and exhausted memory are nobody's
// layout: they stay set, and the call raises them.
static int no(void)
{
    if (PyErr_ExceptionMatches(PyExc_Exception) && !PyErr_ExceptionMatches(PyExc_MemoryError)) PyErr_Clear();
    return 0;
}

static int read_i64(PyObject *o, int64_t *v)
{
    if (!o || !PyLong_CheckExact(o)) return 0;
    *v = PyLong_AsLongLong(o);
    return *v != -1 || !PyErr_Occurred() ? 1 : no();
}

static int read_i32(PyObject *o, int32_t *v)
{
    int64_t w;
    if (!read_i64(o, &w) || w < INT32_MIN || w > INT32_MAX) return 0;
    *v = (int32_t)w;
    return 1;
}

static int read_f32(PyObject *o, float *v)
{
    if (!PyFloat_CheckExact(o)) return 0;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return 1;
}

static int read_ptr(PyObject *t, void **p)                  // None: NULL
{
    *p = NULL;
    if (t == Py_None) return 1;
    PyObject *r = PyObject_VectorcallMethod(s_data_ptr, &t, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
    if (!r) return no();
    if (PyLong_CheckExact(r)) *p = PyLong_AsVoidPtr(r);
    const int ok = PyLong_CheckExact(r) && !PyErr_Occurred();
    Py_DECREF(r);
    return ok ? 1 : no();
}

static int read_pair(PyObject *t, int64_t *a, int64_t *b)   // steals t
{
    if (!t) return no();
    const int ok = PyTuple_Check(t) && PyTuple_GET_SIZE(t) == 2 && read_i64(PyTuple_GET_ITEM(t, 0), a) &&
                   read_i64(PyTuple_GET_ITEM(t, 1), b);
    Py_DECREF(t);
    return ok;
}

// A 2-D operand with a leading dimension: unit stride along a row.
static int read_rows(PyObject *t, void **p, int64_t *ld, int64_t *rows, int64_t *cols)
{
    int64_t unit;
    if (t == Py_None || !read_pair(PyObject_GetAttr(t, s_shape), rows, cols)) return 0;
    if (!read_pair(PyObject_VectorcallMethod(s_stride, &t, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL), ld, &unit)) return 0;
    if ((unit != 1 && *cols > 1) || (*ld < *cols && *rows > 1)) return 0;
    return read_ptr(t, p);
}

static int read_dense(PyObject *t, void **p)
{
    if (t != Py_None) {
        PyObject *r = PyObject_VectorcallMethod(s_is_contiguous, &t, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
        if (!r) return no();
        const int ok = r == Py_True;
        Py_DECREF(r);
        if (!ok) return 0;
    }
    return read_ptr(t, p);
}

static int read_stream(const State *m, mquant_stream_t *s)
{
    if (!m->f_stream) return 0;
    PyObject *r = PyObject_CallNoArgs(m->f_initialized);
    if (!r) return no();
    const int up = r == Py_True;
    Py_DECREF(r);
    if (!up || !(r = PyObject_CallNoArgs(m->f_device))) return no();
    PyObject *st = PyObject_CallOneArg(m->f_stream, r);
    Py_DECREF(r);
    if (!st) return no();
    int ok = PyLong_CheckExact(st);
    if (ok) *s = PyLong_AsVoidPtr(st);
    ok = ok && !PyErr_Occurred();
    Py_DECREF(st);
    return ok ? 1 : no();
}

// ---- operands of the serving entries: of a type, on the current device
static int read_place(const State *m, int64_t *dev, mquant_stream_t *s)
{
    if (!m->f16 || !read_stream(m, s)) return 0;
    PyObject *r = PyObject_CallNoArgs(m->f_device);
    if (!r) return no();
    const int ok = read_i64(r, dev);
    Py_DECREF(r);
    return ok;
}

static int on_device(PyObject *t, int64_t dev)
{
    PyObject *r = PyObject_VectorcallMethod(s_get_device, &t, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, NULL);
    if (!r) return no();
    int64_t at;
    const int ok = read_i64(r, &at) && at == dev;
    Py_DECREF(r);
    return ok;
}

static int placed(PyObject *t, const PyObject *dtype, int64_t dev)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return no();
    Py_DECREF(d);                                              // torch's types live as long as torch
    return d == dtype && on_device(t, dev);
}

static int read_workspace(PyObject *t, int64_t dev, void **p)
{
    return (t == Py_None || on_device(t, dev)) && read_dense(t, p);
}

// `rows` rows (-1: any number, but not none) of at least `cols` columns; the stride of a single row says nothing.
static int read_placed_rows(const State *m, PyObject *t, int64_t dev, int64_t *rows, int64_t cols, void **p, int64_t *ld, int64_t *width)
{
    int64_t r;
    if (!read_rows(t, p, ld, &r, width) || r < 1 || (*rows >= 0 && r != *rows) || *width < cols || !placed(t, m->f16, dev)) return 0;
    if (r == 1) *ld = (*width + 7) & ~(int64_t)7;
    *rows = r;
    return 1;
}

// A contiguous operand of these sizes (-1: any, which is returned); None is NULL where it may be.
static int read_placed(PyObject *t, const PyObject *dtype, int64_t dev, int n, int64_t *shape, int may_miss, void **p)
{
    *p = NULL;
    if (t == Py_None) return may_miss;
    PyObject *s = PyObject_GetAttr(t, s_shape);
    if (!s) return no();
    int ok = PyTuple_Check(s) && PyTuple_GET_SIZE(s) == n;
    for (int i = 0; ok && i < n; ++i) {
        int64_t v = 0;
        ok = read_i64(PyTuple_GET_ITEM(s, i), &v) && (shape[i] < 0 || v == shape[i]);
        shape[i] = v;
    }
    Py_DECREF(s);
    return ok && placed(t, dtype, dev) && read_dense(t, p);
}

// PagedCache.fast: (address of its descriptor, sequences, key/value heads, channels of a head, device)
static int read_cache(PyObject *t, int64_t dev, const mquant_paged_cache_t **c, int64_t *n_seq, int64_t *n_kv, int64_t *head_dim)
{
    int64_t at;
    if (!PyTuple_CheckExact(t) || PyTuple_GET_SIZE(t) != 5) return 0;
    if (!read_i64(PyTuple_GET_ITEM(t, 1), n_seq) || !read_i64(PyTuple_GET_ITEM(t, 2), n_kv) ||
        !read_i64(PyTuple_GET_ITEM(t, 3), head_dim) || !read_i64(PyTuple_GET_ITEM(t, 4), &at) || at != dev)
        return 0;
    *c = PyLong_AsVoidPtr(PyTuple_GET_ITEM(t, 0));
    return PyErr_Occurred() ? no() : 1;
}

static int read_f64(PyObject *o, double *v)
{
    if (!PyFloat_CheckExact(o)) return 0;
    *v = PyFloat_AS_DOUBLE(o);
    return 1;
}

static int read_size(int64_t v, int32_t *out)
{
    *out = (int32_t)v;
    return v >= 0 && v <= INT32_MAX;
}

// (w_prepacked, w_scale, N, out) tuples
static int read_linears(PyObject *list, mquant_linear_t *lin, int32_t *n)
{
    if (!PyList_CheckExact(list) && !PyTuple_CheckExact(list)) return 0;
    const Py_ssize_t len = PySequence_Fast_GET_SIZE(list);
    if (len < 1 || len > 4) return 0;
    for (Py_ssize_t i = 0; i < len; ++i) {
        // a method called below may change the list
        if (PySequence_Fast_GET_SIZE(list) != len) return 0;
        PyObject *t = PySequence_Fast_GET_ITEM(list, i);
        if (!PyTuple_CheckExact(t) || PyTuple_GET_SIZE(t) != 4) return 0;
        Py_INCREF(t);
        void *w, *s, *y;
        int64_t rows, cols;
        const int ok = read_i32(PyTuple_GET_ITEM(t, 2), &lin[i].N) &&
                       read_rows(PyTuple_GET_ITEM(t, 3), &y, &lin[i].ldy, &rows, &cols) &&
                       read_dense(PyTuple_GET_ITEM(t, 1), &s) && read_ptr(PyTuple_GET_ITEM(t, 0), &w);
        Py_DECREF(t);
        if (!ok) return 0;
        lin[i].w_prepacked_dev = w;
        lin[i].w_scale_dev = s;
        lin[i].y_dev = y;
    }
    *n = (int32_t)len;
    return 1;
}

#define SLOW_WAY return slow_way()
static PyObject *slow_way(void)
{
    if (PyErr_Occurred()) return NULL;
    Py_RETURN_NOTIMPLEMENTED;
}

#define LAUNCH(...)                     \
    int st;                             \
    Py_BEGIN_ALLOW_THREADS              \
    st = __VA_ARGS__;                   \
    Py_END_ALLOW_THREADS                \
    return PyLong_FromLong(st)

// ---- entries: the arguments of the functions of binding.py, in order, all positional
static PyObject *prefill_any(const State *m, PyObject *const *a, Py_ssize_t n, int on_scratch)
{
    // x, perm, w_prepacked, w_scale, N, n_vis, s_vis, s_txt, had_block, out [, workspace, its bytes]
    void *x, *perm, *w, *ws, *y, *work = NULL;
    int64_t ldx, ldy, T, K, r, c, bytes = 0;
    int32_t T32, K32, N, n_vis, block;
    float s_vis, s_txt;
    mquant_stream_t s;
    if (n != (on_scratch ? 10 : 12) || !read_rows(a[0], &x, &ldx, &T, &K) || !read_rows(a[9], &y, &ldy, &r, &c) ||
        !read_size(T, &T32) || !read_size(K, &K32) || !read_dense(a[1], &perm) || !read_dense(a[3], &ws) ||
        !read_ptr(a[2], &w) || !read_i32(a[4], &N) || !read_i32(a[5], &n_vis) || !read_f32(a[6], &s_vis) ||
        !read_f32(a[7], &s_txt) || !read_i32(a[8], &block))
        SLOW_WAY;
    if (!on_scratch && (!read_ptr(a[10], &work) || !read_i64(a[11], &bytes))) SLOW_WAY;
    if (!read_stream(m, &s)) SLOW_WAY;
    if (on_scratch) {
        LAUNCH(m->prefill_static(x, ldx, perm, w, ws, y, ldy, T32, N, K32, n_vis, s_vis, s_txt, block, s));
    }
    LAUNCH(m->prefill(x, ldx, perm, w, ws, y, ldy, T32, N, K32, n_vis, s_vis, s_txt, block, work, bytes, s));
}

static PyObject *prefill(PyObject *self, PyObject *const *a, Py_ssize_t n) { return prefill_any(PyModule_GetState(self), a, n, 0); }
static PyObject *prefill_static(PyObject *self, PyObject *const *a, Py_ssize_t n) { return prefill_any(PyModule_GetState(self), a, n, 1); }

static PyObject *decode_grouped(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // x, linears, n_vis, s_vis, s_txt, had_block
    void *x;
    int64_t ldx, T, K;
    int32_t T32, K32, n_vis, block, count;
    float s_vis, s_txt;
    mquant_linear_t lin[4];
    mquant_stream_t s;
    if (n != 6 || !read_rows(a[0], &x, &ldx, &T, &K) || !read_size(T, &T32) || !read_size(K, &K32) ||
        !read_linears(a[1], lin, &count) || !read_i32(a[2], &n_vis) || !read_f32(a[3], &s_vis) ||
        !read_f32(a[4], &s_txt) || !read_i32(a[5], &block) || !read_stream(m, &s))
        SLOW_WAY;
    LAUNCH(m->decode_grouped(x, ldx, T32, K32, n_vis, s_vis, s_txt, block, lin, count, s));
}

static PyObject *decode(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // x, w_prepacked, w_scale, N, n_vis, s_vis, s_txt, had_block, out
    void *x, *w, *ws, *y;
    int64_t ldx, ldy, T, K, r, c;
    int32_t T32, K32, N, n_vis, block;
    float s_vis, s_txt;
    mquant_stream_t s;
    if (n != 9 || !read_rows(a[0], &x, &ldx, &T, &K) || !read_rows(a[8], &y, &ldy, &r, &c) || !read_size(T, &T32) ||
        !read_size(K, &K32) || !read_ptr(a[1], &w) || !read_ptr(a[2], &ws) || !read_i32(a[3], &N) ||
        !read_i32(a[4], &n_vis) || !read_f32(a[5], &s_vis) || !read_f32(a[6], &s_txt) || !read_i32(a[7], &block) ||
        !read_stream(m, &s))
        SLOW_WAY;
    LAUNCH(m->decode(x, ldx, w, ws, y, ldy, T32, N, K32, n_vis, s_vis, s_txt, block, s));
}

static PyObject *gemv_grouped(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // xq, linears, n_vis, s_vis, s_txt
    void *xq;
    int64_t T, K;
    int32_t T32, K32, n_vis, count;
    float s_vis, s_txt;
    mquant_linear_t lin[4];
    mquant_stream_t s;
    if (n != 5 || a[0] == Py_None || !read_pair(PyObject_GetAttr(a[0], s_shape), &T, &K) || !read_dense(a[0], &xq) ||
        !read_size(T, &T32) || !read_size(K, &K32) || !read_linears(a[1], lin, &count) || !read_i32(a[2], &n_vis) ||
        !read_f32(a[3], &s_vis) || !read_f32(a[4], &s_txt) || !read_stream(m, &s))
        SLOW_WAY;
    LAUNCH(m->gemv_grouped(xq, T32, K32, n_vis, s_vis, s_txt, lin, count, s));
}

static PyObject *quant(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // x, n_vis, s_vis, s_txt, had_block, perm, out
    void *x, *perm, *xq;
    int64_t ldx, T, K;
    int32_t T32, K32, n_vis, block;
    float s_vis, s_txt;
    mquant_stream_t s;
    if (n != 7 || !read_rows(a[0], &x, &ldx, &T, &K) || !read_size(T, &T32) || !read_size(K, &K32) ||
        !read_i32(a[1], &n_vis) || !read_f32(a[2], &s_vis) || !read_f32(a[3], &s_txt) || !read_i32(a[4], &block) ||
        !read_dense(a[5], &perm) || !read_dense(a[6], &xq) || !read_stream(m, &s))
        SLOW_WAY;
    LAUNCH(m->quant(x, ldx, perm, xq, T32, K32, n_vis, s_vis, s_txt, block, s));
}

static PyObject *weight_only(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // x, w_prepacked, N, out; an empty x goes the slow way
    void *x, *w, *y;
    int64_t ldx, ldy, T, K, r, c;
    int32_t T32, K32, N;
    mquant_stream_t s;
    if (n != 4 || !read_rows(a[0], &x, &ldx, &T, &K) || !read_rows(a[3], &y, &ldy, &r, &c) || T == 0 ||
        !read_size(T, &T32) || !read_size(K, &K32) || !read_ptr(a[1], &w) || !read_i32(a[2], &N) || !read_stream(m, &s))
        SLOW_WAY;
    LAUNCH(m->weight_only(x, ldx, w, y, ldy, T32, N, K32, s));
}

static PyObject *norm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // q, k, q_weight, k_weight, pos, n_q_heads, n_kv_heads, head_dim, eps, base, q_out, k_out
    void *q, *k, *qw, *kw, *pos, *qo, *ko;
    int64_t dev, T = -1, ldq, ldk, ldqo, ldko, w;
    int32_t T32, n_q, n_kv, D;
    float eps;
    double base;
    mquant_stream_t s;
    if (n != 12 || !read_place(m, &dev, &s) || !read_i32(a[5], &n_q) || !read_i32(a[6], &n_kv) || !read_i32(a[7], &D) || n_q < 1 ||
        n_kv < 1 || D < 1 || !read_f32(a[8], &eps) || !read_f64(a[9], &base))
        SLOW_WAY;
    int64_t one = D;
    if (!read_placed_rows(m, a[0], dev, &T, (int64_t)n_q * D, &q, &ldq, &w) ||
        !read_placed_rows(m, a[1], dev, &T, (int64_t)n_kv * D, &k, &ldk, &w) ||
        !read_placed_rows(m, a[10], dev, &T, (int64_t)n_q * D, &qo, &ldqo, &w) ||
        !read_placed_rows(m, a[11], dev, &T, (int64_t)n_kv * D, &ko, &ldko, &w) || !read_size(T, &T32) ||
        !read_placed(a[2], m->f16, dev, 1, &one, 1, &qw) || !read_placed(a[3], m->f16, dev, 1, &one, 1, &kw) ||
        !read_placed(a[4], m->i32, dev, 1, &T, 0, &pos))
        SLOW_WAY;
    LAUNCH(m->norm(q, ldq, qo, ldqo, k, ldk, ko, ldko, qw, kw, eps, pos, T32, n_q, n_kv, D, base, s));
}

static PyObject *append(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // q, k, v, cache, row_start, pos, n_q_heads, q_weight, k_weight, eps, base, rope_pos, q_out
    void *q, *k, *v, *qw, *kw, *start, *pos, *rope, *qo;
    const mquant_paged_cache_t *c;
    int64_t dev, T = -1, ldq, ldk, ldv, ldqo, w, n_seq, n_kv, D;
    int32_t T32, n_q;
    float eps;
    double base;
    mquant_stream_t s;
    if (n != 13 || !read_place(m, &dev, &s) || !read_cache(a[3], dev, &c, &n_seq, &n_kv, &D) || !read_i32(a[6], &n_q) || n_q < 1 ||
        !read_f32(a[9], &eps) || !read_f64(a[10], &base))
        SLOW_WAY;
    int64_t starts = n_seq + 1, one = D;
    if (!read_placed_rows(m, a[0], dev, &T, n_q * D, &q, &ldq, &w) || !read_placed_rows(m, a[1], dev, &T, n_kv * D, &k, &ldk, &w) ||
        !read_placed_rows(m, a[2], dev, &T, n_kv * D, &v, &ldv, &w) || !read_placed_rows(m, a[12], dev, &T, n_q * D, &qo, &ldqo, &w) ||
        !read_size(T, &T32) || !read_placed(a[4], m->i32, dev, 1, &starts, 0, &start) || !read_placed(a[5], m->i32, dev, 1, &T, 0, &pos) ||
        !read_placed(a[7], m->f16, dev, 1, &one, 1, &qw) || !read_placed(a[8], m->f16, dev, 1, &one, 1, &kw) ||
        !read_placed(a[11], m->i32, dev, 1, &T, 1, &rope))
        SLOW_WAY;
    LAUNCH(m->append(q, ldq, qo, ldqo, k, ldk, v, ldv, qw, kw, eps, start, pos, rope, T32, n_q, base, c, s));
}

static PyObject *attention(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // q, cache, row_start, pos, n_q_heads, max_rows, max_kv, out, workspace, its bytes
    void *q, *start, *pos, *o, *work;
    const mquant_paged_cache_t *c;
    int64_t dev, T = -1, ldq, ldo, w, n_seq, n_kv, D, bytes;
    int32_t T32, n_q, max_rows, max_kv;
    mquant_stream_t s;
    if (n != 10 || !read_place(m, &dev, &s) || !read_cache(a[1], dev, &c, &n_seq, &n_kv, &D) || !read_i32(a[4], &n_q) || n_q < 1 ||
        !read_i32(a[5], &max_rows) || !read_i32(a[6], &max_kv) || !read_i64(a[9], &bytes))
        SLOW_WAY;
    int64_t starts = n_seq + 1;
    if (!read_placed_rows(m, a[0], dev, &T, n_q * D, &q, &ldq, &w) || !read_placed_rows(m, a[7], dev, &T, n_q * D, &o, &ldo, &w) ||
        !read_size(T, &T32) || !read_placed(a[2], m->i32, dev, 1, &starts, 0, &start) || !read_placed(a[3], m->i32, dev, 1, &T, 0, &pos) ||
        !read_workspace(a[8], dev, &work))
        SLOW_WAY;
    LAUNCH(m->attention(q, ldq, c, start, pos, o, ldo, T32, n_q, max_rows, max_kv, work, bytes, s));
}

static PyObject *lora(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    const State *m = PyModule_GetState(self);
    // x, adapter, a, b, scale, base, perm, out, workspace, its bytes
    void *x, *id, *pa, *pb, *scale, *base, *perm, *y, *work;
    int64_t dev, T = -1, ldx, ldb, ldy, K, N, wy, bytes, count = -1;
    int32_t T32, N32, K32, rank32, n32;
    mquant_stream_t s;
    if (n != 10 || !read_place(m, &dev, &s) || !read_placed_rows(m, a[0], dev, &T, 0, &x, &ldx, &K) ||
        !read_placed_rows(m, a[5], dev, &T, 0, &base, &ldb, &N) || !read_placed_rows(m, a[7], dev, &T, N, &y, &ldy, &wy) || wy != N ||
        !read_i64(a[9], &bytes))
        SLOW_WAY;
    int64_t sa[3] = {-1, -1, K};
    if (!read_placed(a[2], m->f16, dev, 3, sa, 0, &pa)) SLOW_WAY;
    int64_t sb[3] = {sa[0], N, sa[1]};
    count = sa[0];
    if (!read_placed(a[3], m->f16, dev, 3, sb, 0, &pb) || !read_placed(a[4], m->f32, dev, 1, &count, 0, &scale) ||
        !read_placed(a[1], m->i32, dev, 1, &T, 0, &id) || !read_placed(a[6], m->i32, dev, 1, &T, 1, &perm) ||
        !read_workspace(a[8], dev, &work) ||
        !read_size(T, &T32) || !read_size(N, &N32) || !read_size(K, &K32) || !read_size(sa[1], &rank32) || !read_size(count, &n32))
        SLOW_WAY;
    LAUNCH(m->lora(x, ldx, perm, id, pa, pb, scale, base, ldb, y, ldy, T32, N32, K32, rank32, n32, work, bytes, s));
}

// setup_serving(float16, float32, int32, addresses of the four entries in the order of State), behind setup()
static PyObject *setup_serving(PyObject *self, PyObject *args)
{
    PyObject *f16, *f32, *i32, *addr[4];
    if (!PyArg_ParseTuple(args, "OOOO!O!O!O!", &f16, &f32, &i32, &PyLong_Type, &addr[0], &PyLong_Type, &addr[1], &PyLong_Type, &addr[2],
                          &PyLong_Type, &addr[3]))
        return NULL;
    void *p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(addr[i]);
        if (PyErr_Occurred()) return NULL;
    }
    State *m = PyModule_GetState(self);
    *(void **)&m->norm = p[0];
    *(void **)&m->append = p[1];
    *(void **)&m->attention = p[2];
    *(void **)&m->lora = p[3];
    Py_INCREF(f16), Py_INCREF(f32), Py_INCREF(i32);
    Py_XSETREF(m->f32, f32);
    Py_XSETREF(m->i32, i32);
    Py_XSETREF(m->f16, f16);
    Py_RETURN_NONE;
}

// setup(is_initialized, device, raw stream, addresses of the seven entries of the library in the order of State)
static PyObject *setup(PyObject *self, PyObject *args)
{
    PyObject *init, *dev, *st, *addr[7];
    if (!PyArg_ParseTuple(args, "OOOO!O!O!O!O!O!O!", &init, &dev, &st, &PyLong_Type, &addr[0], &PyLong_Type, &addr[1],
                          &PyLong_Type, &addr[2], &PyLong_Type, &addr[3], &PyLong_Type, &addr[4], &PyLong_Type, &addr[5],
                          &PyLong_Type, &addr[6]))
        return NULL;
    void *p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(addr[i]);
        if (PyErr_Occurred()) return NULL;
    }
    State *m = PyModule_GetState(self);
    *(void **)&m->prefill = p[0];
    *(void **)&m->prefill_static = p[1];
    *(void **)&m->decode = p[2];
    *(void **)&m->decode_grouped = p[3];
    *(void **)&m->gemv_grouped = p[4];
    *(void **)&m->quant = p[5];
    *(void **)&m->weight_only = p[6];
    Py_INCREF(init), Py_INCREF(dev), Py_INCREF(st);
    Py_XSETREF(m->f_initialized, init);
    Py_XSETREF(m->f_device, dev);
    Py_XSETREF(m->f_stream, st);
    Py_RETURN_NONE;
}

#define ENTRY(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    ENTRY(prefill), ENTRY(prefill_static), ENTRY(decode), ENTRY(decode_grouped), ENTRY(gemv_grouped), ENTRY(quant),
    ENTRY(weight_only), ENTRY(norm), ENTRY(append), ENTRY(attention), ENTRY(lora), {"setup", setup, METH_VARARGS, NULL},
    {"setup_serving", setup_serving, METH_VARARGS, NULL}, {NULL, NULL, 0, NULL},
};

static int traverse(PyObject *self, visitproc visit, void *arg)
{
    State *m = PyModule_GetState(self);
    Py_VISIT(m->f_initialized);
    Py_VISIT(m->f_device);
    Py_VISIT(m->f_stream);
    Py_VISIT(m->f16);
    Py_VISIT(m->f32);
    Py_VISIT(m->i32);
    return 0;
}

static int clear(PyObject *self)
{
    State *m = PyModule_GetState(self);
    Py_CLEAR(m->f_stream);                     // first: a module without it takes no call
    Py_CLEAR(m->f_initialized);
    Py_CLEAR(m->f_device);
    Py_CLEAR(m->f16);
    Py_CLEAR(m->f32);
    Py_CLEAR(m->i32);
    return 0;
}

static int start(PyObject *self)
{
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    return s_shape && s_stride && s_data_ptr && s_is_contiguous && s_dtype && s_get_device ? 0 : -1;
}

static PyModuleDef_Slot slots[] = {{Py_mod_exec, start}, {0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "mquant_fastcall", NULL, sizeof(State), methods, slots, traverse,
                                    clear, NULL};

PyMODINIT_FUNC PyInit_mquant_fastcall(void) { return PyModuleDef_Init(&module); }
