/*
 * The Python side of gspc_conv2d_grouped, and of the channels-last operators: argument marshalling in C.
 *
 * A call of the library for a small layer is a launch of 3-4 us on the GPU; through ctypes, which converts
 * thirteen arguments by type and builds an object for each pointer, the call took 4.6 us of host time, 2.5-2.8 of them
 * in Python (64 -> 64 on 32x32, g = 4, N = 1).  Here they are 0.4, and the call takes 3.8 in all.  The library is not
 * linked: binding.py hands over the address of the function that it loaded.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*conv_fn)(const void *, const void *, int, int, int, int, int, int, int, int, int, int, void *);

static conv_fn g_conv = NULL;
static PyObject *s_data_ptr, *s_value;

static PyObject *bind(PyObject *self, PyObject *arg) {
    (void)self;
    void *p = PyLong_AsVoidPtr(arg);
    if (!p && PyErr_Occurred()) return NULL;
    g_conv = (conv_fn)p;
    Py_RETURN_NONE;
}

/* tensor.data_ptr(), NULL for None.  0: done, -1: exception. */
static int tensor_ptr(PyObject *t, void **out) {
    if (t == Py_None) {
        *out = NULL;
        return 0;
    }
    PyObject *v = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!v) return -1;
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    return !*out && PyErr_Occurred() ? -1 : 0;
}

/* conv(input, handle, N, Cin, H, W, Cout, KH, KW, stride, pad, groups, output) -> status code, or NotImplemented where an
 * argument is of a kind that only the general route converts (a number that is not a plain int, or does not fit one). */
static PyObject *conv(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    if (n != 13 || !g_conv) Py_RETURN_NOTIMPLEMENTED;
    int v[10];
    for (int i = 0; i < 10; ++i) {
        if (!PyLong_CheckExact(a[2 + i])) Py_RETURN_NOTIMPLEMENTED;
        int over;
        const long x = PyLong_AsLongAndOverflow(a[2 + i], &over);
        if (over || x != (int)x) Py_RETURN_NOTIMPLEMENTED;
        v[i] = (int)x;
    }
    void *in, *w = NULL, *out;
    if (a[1] != Py_None) {
        PyObject *h = PyObject_GetAttr(a[1], s_value);     /* a ctypes.c_void_p */
        if (!h) {
            PyErr_Clear();
            Py_RETURN_NOTIMPLEMENTED;
        }
        const int plain = h == Py_None || PyLong_CheckExact(h);
        if (plain && h != Py_None) w = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!plain) Py_RETURN_NOTIMPLEMENTED;
        if (!w && PyErr_Occurred()) return NULL;
    }
    if (tensor_ptr(a[0], &in) || tensor_ptr(a[12], &out)) return NULL;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_conv(in, w, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], out);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* ---- channels-last operators -----------------------------------------------------------------------------------------
 * The same for their calls with everything given: contiguous tensors on the GPU of the types and sizes that fit one another.  Whatever
 * else there is - an output to be made, rows with gaps, a mistake - is NotImplemented, and the general route's. */
typedef int (*layout_fn)(const void *, int, int, int, int, void *, int);
typedef int (*quantize_fn)(const void *, int, int64_t, int64_t, int, void *, float *);
typedef int (*dequantize_fn)(const void *, const float *, int64_t, int, void *, int, int64_t);
typedef int (*norm_fn)(const void *, int, int64_t, const float *, const float *, int, int, int, int, float, int, void *, int, int64_t, float *,
                       float *, void *, float *, void *, size_t);
typedef int (*norm_backward_fn)(const void *, int, int64_t, const void *, int, int64_t, const float *, const float *, const float *,
                                const float *, int, int, int, int, int, void *, int64_t, float *, float *, void *, size_t);
typedef int (*matmul_fn)(const void *, const float *, const void *, const float *, const float *, int64_t, int, int, void *, int, int64_t);

static struct {
    layout_fn pack, unpack;
    quantize_fn quantize;
    dequantize_fn dequantize;
    norm_fn norm;
    norm_backward_fn norm_backward;
    matmul_fn matmul;
} g_calls;
static PyObject *g_types[6];               /* torch.float32, bfloat16, int8, float8_e4m3fn, in the order of the library's numbers; uint8, int64 */
enum { F32, BF16, I8, F8, U8, I64, TYPES };
static PyObject *s_is_cuda, *s_dtype, *s_shape, *s_is_contiguous;

static PyObject *bind_tokens(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    if (n != 10) {
        PyErr_SetString(PyExc_TypeError, "seven addresses and three types");
        return NULL;
    }
    void *p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i] && PyErr_Occurred()) return NULL;
    }
    g_calls.pack = (layout_fn)p[0];
    g_calls.unpack = (layout_fn)p[1];
    g_calls.quantize = (quantize_fn)p[2];
    g_calls.dequantize = (dequantize_fn)p[3];
    g_calls.norm = (norm_fn)p[4];
    g_calls.norm_backward = (norm_backward_fn)p[5];
    g_calls.matmul = (matmul_fn)p[6];
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[7 + i]);
        g_types[i] = a[7 + i];
    }
    Py_RETURN_NONE;
}

typedef struct {
    void *ptr;
    int type, dims;
    int64_t first, second, last, count;    /* first, second and last dimension, elements */
} tensor_t;

static int is_true(PyObject *v) {
    const int yes = v == Py_True;
    Py_XDECREF(v);
    return yes;
}

/* A contiguous tensor on the GPU of one of the types.  0: not one (no exception is left). */
static int tensor_of_any(PyObject *t, tensor_t *o) {
    if (!is_true(PyObject_GetAttr(t, s_is_cuda))) goto no;
    PyObject *v = PyObject_GetAttr(t, s_dtype);
    if (!v) goto no;
    for (o->type = 0; o->type < TYPES && v != g_types[o->type]; ++o->type) {}
    Py_DECREF(v);
    if (o->type == TYPES || !is_true(PyObject_CallMethodNoArgs(t, s_is_contiguous))) goto no;
    v = PyObject_GetAttr(t, s_shape);
    if (!v || !PyTuple_Check(v)) {
        Py_XDECREF(v);
        goto no;
    }
    o->dims = (int)PyTuple_GET_SIZE(v);
    o->count = 1;
    o->first = o->second = o->last = 1;
    for (int i = 0; i < o->dims; ++i) {
        o->last = PyLong_AsLongLong(PyTuple_GET_ITEM(v, i));
        if (i == 0) o->first = o->last;
        if (i == 1) o->second = o->last;
        o->count *= o->last;
    }
    Py_DECREF(v);
    return !PyErr_Occurred() && !tensor_ptr(t, &o->ptr);
no:
    PyErr_Clear();
    return 0;
}
/* One of the first three. */
static int tensor(PyObject *t, tensor_t *o) { return tensor_of_any(t, o) && o->type <= I8; }
/* One of a type and of a number of elements, or NULL where none is allowed. */
static int vector(PyObject *t, int type, int64_t count, int none, void **ptr) {
    tensor_t o;
    *ptr = NULL;
    if (t == Py_None) return none;
    if (!tensor_of_any(t, &o) || o.type != type || o.count != count) return 0;
    *ptr = o.ptr;
    return 1;
}
/* 8-bit rows: a pair of int8 [rows * pitch] and fp32 [rows]. */
static int rows8(PyObject *t, int64_t rows, int64_t cols, void **q, void **scale) {
    return PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 2 && vector(PyTuple_GET_ITEM(t, 0), 2, rows * ((cols + 15) / 16 * 16), 0, q) &&
           vector(PyTuple_GET_ITEM(t, 1), 0, rows, 0, scale);
}
static int small(PyObject *v, int *out) {
    if (!PyLong_CheckExact(v)) return 0;
    int over;
    const long x = PyLong_AsLongAndOverflow(v, &over);
    *out = (int)x;
    return !over && x == (int)x;
}
static int fits(int64_t v) { return v > 0 && v < 0x7ffffff0; }

#define GENERAL                      \
    do {                             \
        PyErr_Clear();               \
        Py_RETURN_NOTIMPLEMENTED;    \
    } while (0)
#define CALL(expression)             \
    int rc;                          \
    Py_BEGIN_ALLOW_THREADS           \
    rc = expression;                 \
    Py_END_ALLOW_THREADS             \
    return PyLong_FromLong(rc)

/* pack(x [N, C, P], out [N, ..., C] or [N * P, C]), unpack(x [N, P, C], out [N, C, ...]) */
static PyObject *layout(PyObject *const *a, Py_ssize_t n, int pack) {
    tensor_t x, out;
    if (n != 2 || !g_calls.pack || !tensor(a[0], &x) || x.dims != 3 || !fits(x.count) || x.type == 2 || !tensor(a[1], &out) || out.type == 2 ||
        out.count != x.count || out.dims < (pack ? 2 : 3) || (out.dims > 2 && out.first != x.first) || (pack ? out.last != x.second : out.second != x.last))
        GENERAL;
    const int N = (int)x.first, C = (int)(pack ? x.second : x.last);
    CALL((pack ? g_calls.pack : g_calls.unpack)(x.ptr, x.type, N, C, (int)(x.count / N / C), out.ptr, out.type));
}
static PyObject *pack(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    return layout(a, n, 1);
}
static PyObject *unpack(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    return layout(a, n, 0);
}

/* quantize(x [..., cols], (q, scale)) */
static PyObject *quantize(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x;
    void *q, *scale;
    if (n != 2 || !g_calls.quantize || !tensor(a[0], &x) || x.type == 2 || !fits(x.last) || !rows8(a[1], x.count / x.last, x.last, &q, &scale)) GENERAL;
    CALL(g_calls.quantize(x.ptr, x.type, x.last, x.count / x.last, (int)x.last, q, scale));
}

/* dequantize((q, scale), cols, out [..., cols]) */
static PyObject *dequantize(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x;
    void *q, *scale;
    int cols;
    if (n != 3 || !g_calls.dequantize || !small(a[1], &cols) || !tensor(a[2], &x) || x.type == 2 || cols <= 0 || x.last != cols ||
        !rows8(a[0], x.count / cols, cols, &q, &scale))
        GENERAL;
    CALL(g_calls.dequantize(q, scale, x.count / cols, cols, x.ptr, x.type, cols));
}

static size_t bytes_of(const tensor_t *t) { return t->ptr ? (size_t)t->count * (t->type == I64 ? 8 : t->type == F32 ? 4 : t->type == BF16 ? 2 : 1) : 0; }

/* Whether two tensors of up to four dimensions (more: no) have the same shape. */
static int same_shape(const tensor_t *a, const tensor_t *b) {
    return a->dims == b->dims && a->dims <= 4 && a->first == b->first && a->second == b->second && a->last == b->last && a->count == b->count;
}

/* norm(x [N, ..., C], gamma, beta, groups, eps, act, out, stats, saved, workspace) */
static PyObject *norm(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x, y, ws = {0};
    void *gamma, *beta, *stats, *out, *scale = NULL, *saved = NULL, *saved_scale = NULL;
    int groups, act, kind;
    if (n != 10 || !g_calls.norm || !tensor(a[0], &x) || x.type == 2 || x.dims < 3 || !fits(x.first) || !fits(x.last) || !small(a[3], &groups) ||
        !PyFloat_CheckExact(a[4]) || !small(a[5], &act) || !fits(x.count / x.first / x.last) || !vector(a[1], 0, x.last, 1, &gamma) ||
        !vector(a[2], 0, x.last, 1, &beta) || !vector(a[7], 0, x.first * groups * 2, 1, &stats) || (a[9] != Py_None && !tensor(a[9], &ws)))
        GENERAL;
    const int64_t rows = x.count / x.last;
    if (PyTuple_CheckExact(a[6])) {
        if (!rows8(a[6], rows, x.last, &out, &scale)) GENERAL;
        kind = 2;
    } else {
        if (!tensor(a[6], &y) || y.type == 2 || !same_shape(&y, &x)) GENERAL;
        out = y.ptr;
        kind = y.type;
    }
    if (a[8] != Py_None && !rows8(a[8], rows, x.last, &saved, &saved_scale)) GENERAL;
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    CALL(g_calls.norm(x.ptr, x.type, x.last, gamma, beta, (int)x.first, (int)(rows / x.first), (int)x.last, groups, eps, act, out, kind, x.last, scale,
                      stats, saved, saved_scale, ws.ptr, bytes_of(&ws)));
}

/* norm_backward(dy [N, ..., C], x, stats, gamma, beta, groups, act, dx, dgamma, dbeta, workspace) */
static PyObject *norm_backward(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t dy, x, dx, ws = {0};
    void *gamma, *beta, *stats, *dgamma, *dbeta, *px, *scale = NULL;
    int groups, act, kind;
    if (n != 11 || !g_calls.norm_backward || !tensor(a[0], &dy) || dy.type == 2 || dy.dims < 3 || !fits(dy.first) || !fits(dy.last) ||
        !fits(dy.count / dy.first / dy.last) || !small(a[5], &groups) || !small(a[6], &act) || !vector(a[2], 0, dy.first * groups * 2, 0, &stats) ||
        !vector(a[3], 0, dy.last, 1, &gamma) || !vector(a[4], 0, dy.last, 1, &beta) || !vector(a[8], 0, dy.last, 0, &dgamma) ||
        !vector(a[9], 0, dy.last, 0, &dbeta) || !tensor(a[7], &dx) || dx.type != dy.type || !same_shape(&dx, &dy) ||
        (a[10] != Py_None && !tensor(a[10], &ws)))
        GENERAL;
    const int64_t rows = dy.count / dy.last;
    if (PyTuple_CheckExact(a[1])) {
        if (!rows8(a[1], rows, dy.last, &px, &scale)) GENERAL;
        kind = 2;
    } else {
        if (!tensor(a[1], &x) || x.type == 2 || !same_shape(&x, &dy)) GENERAL;
        px = x.ptr;
        kind = x.type;
    }
    CALL(g_calls.norm_backward(dy.ptr, dy.type, dy.last, px, kind, dy.last, scale, stats, gamma, beta, (int)dy.first, (int)(rows / dy.first),
                               (int)dy.last, groups, act, dx.ptr, dy.last, dgamma, dbeta, ws.ptr, bytes_of(&ws)));
}

/* matmul((q, scale), (q, scale), bias, out [..., N], cols = None: all of the pitch) */
static PyObject *matmul(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x, w, out;
    void *sa, *sw, *bias;
    int cols = 0;
    if (n < 4 || n > 5 || (n == 5 && a[4] != Py_None && (!small(a[4], &cols) || cols <= 0)) || !g_calls.matmul || !PyTuple_CheckExact(a[0]) || PyTuple_GET_SIZE(a[0]) != 2 || !PyTuple_CheckExact(a[1]) ||
        PyTuple_GET_SIZE(a[1]) != 2 || !tensor(PyTuple_GET_ITEM(a[0], 0), &x) || !tensor(PyTuple_GET_ITEM(a[1], 0), &w) || x.type != 2 ||
        w.type != 2 || x.dims != 2 || w.dims != 2 || x.last != w.last || x.last % 16 || !fits(x.last) || (cols && (cols + (int64_t)15) / 16 * 16 != x.last) || !fits(w.first) ||
        !vector(PyTuple_GET_ITEM(a[0], 1), 0, x.first, 0, &sa) || !vector(PyTuple_GET_ITEM(a[1], 1), 0, w.first, 0, &sw) ||
        !vector(a[2], 0, w.first, 1, &bias) || !tensor(a[3], &out) || out.type == 2 || out.last != w.first || out.count != x.first * w.first)
        GENERAL;
    CALL(g_calls.matmul(x.ptr, sa, w.ptr, sw, bias, x.first, (int)w.first, cols ? cols : (int)x.last, out.ptr, out.type, w.first));
}

/* ---- a residual block on tokens: the same ---------------------------------------------------------------------------- */
typedef struct {
    int64_t rows, gates;
    int cols, post, pre, act;
    void *post_gamma, *post_beta, *pre_gamma, *pre_beta, *gate;
    float scale, eps;
    double drop;
    uint64_t seed, offset;
    void *step;
} residual_t;                       /* gspc_residual_t */
typedef int (*quantize_f8_fn)(const void *, int, int64_t, int64_t, int, void *, void *, void *, void *);
typedef int (*dequantize_f8_fn)(const void *, const void *, int64_t, int, void *, int, int64_t);
typedef int (*matmul_f8_fn)(const void *, const void *, const void *, const void *, const void *, int64_t, int, int, void *, int, int64_t, void *, size_t);
typedef int (*dropout_fn)(const void *, int, int64_t, int64_t, int, double, uint64_t, uint64_t, const void *, void *, int64_t);
typedef int (*residual_norm_fn)(const residual_t *, const void *, int, int64_t, const void *, int, int64_t, void *, int64_t, void *, int, int64_t, void *, void *);
typedef int (*residual_norm_backward_fn)(const residual_t *, const void *, int, int64_t, const void *, int64_t, const void *, int, int64_t, const void *, int,
                                         int64_t, const void *, void *, int64_t, void *, int64_t, void *, void *, void *, void *, void *, void *, size_t);
static struct {
    quantize_f8_fn quantize;
    dequantize_f8_fn dequantize;
    matmul_f8_fn matmul;
    dropout_fn dropout;
    residual_norm_fn residual_norm;
    residual_norm_backward_fn residual_norm_backward;
    size_t (*matmul_bytes)(int64_t, int, int);
    size_t (*residual_norm_backward_bytes)(int64_t, int, int64_t);
} g_block;

static PyObject *bind_block(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "eight addresses and three types");
        return NULL;
    }
    void *p[8];
    for (int i = 0; i < 8; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i] && PyErr_Occurred()) return NULL;
    }
    g_block.quantize = (quantize_f8_fn)p[0];
    g_block.dequantize = (dequantize_f8_fn)p[1];
    g_block.matmul = (matmul_f8_fn)p[2];
    g_block.dropout = (dropout_fn)p[3];
    g_block.residual_norm = (residual_norm_fn)p[4];
    g_block.residual_norm_backward = (residual_norm_backward_fn)p[5];
    g_block.matmul_bytes = (size_t (*)(int64_t, int, int))p[6];
    g_block.residual_norm_backward_bytes = (size_t (*)(int64_t, int, int64_t))p[7];
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[8 + i]);
        g_types[F8 + i] = a[8 + i];
    }
    Py_RETURN_NONE;
}

/* 8-bit float rows: a pair of e4m3 [rows * pitch] and uint8 [rows * scale pitch]. */
static int rows_f8(PyObject *t, int64_t rows, int64_t cols, void **q, void **scale) {
    return PyTuple_CheckExact(t) && PyTuple_GET_SIZE(t) == 2 && vector(PyTuple_GET_ITEM(t, 0), F8, rows * ((cols + 127) / 128 * 128), 0, q) &&
           vector(PyTuple_GET_ITEM(t, 1), U8, rows * ((cols + 511) / 512 * 4), 0, scale);
}
static int word(PyObject *v, uint64_t *out) {
    if (!PyLong_CheckExact(v)) return 0;
    *out = PyLong_AsUnsignedLongLong(v);
    return !PyErr_Occurred();
}
static int real(PyObject *v, double *out) {
    if (!PyFloat_CheckExact(v)) return 0;
    *out = PyFloat_AS_DOUBLE(v);
    return 1;
}
static int is_dense(PyObject *t, tensor_t *o) { return tensor_of_any(t, o) && o->type <= BF16; }
static int fits_f8(int64_t v) { return v > 0 && v <= 0x7ffffc00; }

/* The workspace of a call: the caller's (`given`, a tensor or None), or what make(bytes, like) returns where some are needed.  0: what is given is
 * no workspace; -1: an exception. */
static int workspace(PyObject *given, size_t need, PyObject *make, PyObject *like, tensor_t *ws, PyObject **held) {
    *held = NULL;
    ws->ptr = NULL;
    if (given != Py_None) return tensor_of_any(given, ws);
    if (!need) return 1;
    PyObject *bytes = PyLong_FromSize_t(need);
    if (!bytes) return -1;
    *held = PyObject_CallFunctionObjArgs(make, bytes, like, NULL);
    Py_DECREF(bytes);
    if (!*held) return -1;
    return tensor_of_any(*held, ws);
}
#define CALL_WITH(held, expression)  \
    int rc;                          \
    Py_BEGIN_ALLOW_THREADS           \
    rc = expression;                 \
    Py_END_ALLOW_THREADS             \
    Py_XDECREF(held);                \
    return PyLong_FromLong(rc)

/* quantize_f8(x [..., cols], (q, scale) or None, (qt, scale_t) or None) */
static PyObject *quantize_f8(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x;
    void *q = NULL, *scale = NULL, *qt = NULL, *scale_t = NULL;
    if (n != 3 || !g_block.quantize || !is_dense(a[0], &x) || !fits_f8(x.last) || !fits_f8(x.count / x.last)) GENERAL;
    const int64_t rows = x.count / x.last;
    if ((a[1] != Py_None && !rows_f8(a[1], rows, x.last, &q, &scale)) || (a[2] != Py_None && !rows_f8(a[2], x.last, rows, &qt, &scale_t))) GENERAL;
    CALL(g_block.quantize(x.ptr, x.type, x.last, rows, (int)x.last, q, scale, qt, scale_t));
}

/* dequantize_f8((q, scale), cols, out [..., cols]) */
static PyObject *dequantize_f8(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x;
    void *q, *scale;
    int cols;
    if (n != 3 || !g_block.dequantize || !small(a[1], &cols) || !is_dense(a[2], &x) || !fits_f8(cols) || x.last != cols ||
        !rows_f8(a[0], x.count / cols, cols, &q, &scale))
        GENERAL;
    CALL(g_block.dequantize(q, scale, x.count / cols, cols, x.ptr, x.type, cols));
}

/* matmul_f8((q, scale), (q, scale), bias, out [..., N], cols or None: all of the pitch, workspace, make) */
static PyObject *matmul_f8(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x, w, out, ws = {0};
    void *sa, *sw, *bias;
    int cols = 0;
    if (n != 7 || (a[4] != Py_None && (!small(a[4], &cols) || cols <= 0)) || !g_block.matmul || !PyTuple_CheckExact(a[0]) || PyTuple_GET_SIZE(a[0]) != 2 ||
        !PyTuple_CheckExact(a[1]) || PyTuple_GET_SIZE(a[1]) != 2 || !tensor_of_any(PyTuple_GET_ITEM(a[0], 0), &x) ||
        !tensor_of_any(PyTuple_GET_ITEM(a[1], 0), &w) || x.type != F8 || w.type != F8 || x.dims != 2 || w.dims != 2 || x.last != w.last || x.last % 128 ||
        !fits_f8(x.last) || (cols && (cols + (int64_t)127) / 128 * 128 != x.last) || !fits(w.first) ||
        !vector(PyTuple_GET_ITEM(a[0], 1), U8, x.first * ((x.last + 511) / 512 * 4), 0, &sa) ||
        !vector(PyTuple_GET_ITEM(a[1], 1), U8, w.first * ((x.last + 511) / 512 * 4), 0, &sw) || !vector(a[2], F32, w.first, 1, &bias) ||
        !is_dense(a[3], &out) || out.last != w.first || out.count != x.first * w.first)
        GENERAL;
    PyObject *held;
    const int ok = workspace(a[5], a[5] == Py_None ? g_block.matmul_bytes(x.first, (int)w.first, (int)x.last) : 0, a[6], a[3], &ws, &held);
    if (ok < 0) return NULL;
    if (!ok) {
        Py_XDECREF(held);
        GENERAL;
    }
    CALL_WITH(held, g_block.matmul(x.ptr, sa, w.ptr, sw, bias, x.first, (int)w.first, (int)x.last, out.ptr, out.type, w.first, ws.ptr, bytes_of(&ws)));
}

/* dropout(x [..., cols], drop, seed, offset, step, out) */
static PyObject *dropout(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x, out;
    double drop;
    uint64_t seed, offset;
    void *step;
    if (n != 6 || !g_block.dropout || !is_dense(a[0], &x) || !real(a[1], &drop) || !word(a[2], &seed) || !word(a[3], &offset) ||
        !vector(a[4], I64, 1, 1, &step) || !is_dense(a[5], &out) || out.type != x.type || !same_shape(&out, &x) || !fits(x.last))
        GENERAL;
    CALL(g_block.dropout(x.ptr, x.type, x.last, x.count / x.last, (int)x.last, drop, seed, offset, step, out.ptr, x.last));
}

/* What the forward call and the gradient have in common: gate, post, its parameters, pre, its parameters, act, scale; then drop, seed, offset, step. */
static int residual(PyObject *const *a, PyObject *const *b, int64_t rows, int64_t cols, residual_t *r) {
    double scale;
    tensor_t gate;
    r->rows = rows;
    r->cols = (int)cols;
    r->gates = 1;
    r->gate = NULL;
    if (a[0] != Py_None) {
        if (!tensor_of_any(a[0], &gate) || gate.type != F32 || gate.last != cols) return 0;
        r->gate = gate.ptr;
        r->gates = gate.count / cols;
    }
    if (!small(a[1], &r->post) || !vector(a[2], F32, cols, 1, &r->post_gamma) || !vector(a[3], F32, cols, 1, &r->post_beta) || !small(a[4], &r->pre) ||
        !vector(a[5], F32, cols, 1, &r->pre_gamma) || !vector(a[6], F32, cols, 1, &r->pre_beta) || !small(a[7], &r->act) || !real(a[8], &scale) ||
        !real(b[0], &r->drop) || !word(b[1], &r->seed) || !word(b[2], &r->offset) || !vector(b[3], I64, 1, 1, &r->step))
        return 0;
    r->scale = (float)scale;
    return 1;
}
/* A dense tensor of a type (-1: of either) and of the shape of another, or none. */
static int alike(PyObject *t, const tensor_t *of, int type, tensor_t *o) {
    o->ptr = NULL;
    o->type = F32;
    return t == Py_None || (is_dense(t, o) && (type < 0 || o->type == type) && same_shape(o, of));
}

/* residual_norm(x, h, gate, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, act, scale, eps, drop, seed, offset, step, xo, out, stats) */
static PyObject *residual_norm(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t x, h, xo, z = {0};
    residual_t r;
    double eps;
    void *stats, *z_scale = NULL;
    if (n != 19 || !g_block.residual_norm || !is_dense(a[0], &x) || x.last <= 0 || x.last > 8192 || !alike(a[1], &x, -1, &h) || !real(a[11], &eps) ||
        !alike(a[16], &x, x.type, &xo))
        GENERAL;
    const int64_t rows = x.count / x.last;
    if (!residual(a + 2, a + 12, rows, x.last, &r) || !vector(a[18], F32, rows * 4, 1, &stats)) GENERAL;
    if (PyTuple_CheckExact(a[17])) {
        if (!rows_f8(a[17], rows, x.last, &z.ptr, &z_scale)) GENERAL;
        z.type = F8;
    } else if (a[17] == Py_None || !alike(a[17], &x, -1, &z))
        GENERAL;
    r.eps = (float)eps;
    CALL(g_block.residual_norm(&r, x.ptr, x.type, x.last, h.ptr, h.type, x.last, xo.ptr, x.last, z.ptr, z.type, x.last, z_scale, stats));
}

/* residual_norm_backward(dz, dxo, xo, h, stats, gate, post, post_gamma, post_beta, pre, pre_gamma, pre_beta, act, scale, drop, seed, offset, step, dx, dh,
 * dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta, workspace, make) */
static PyObject *residual_norm_backward(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    (void)self;
    tensor_t dz, dxo, xo, h, dx, dh, ws = {0};
    residual_t r;
    void *stats, *g[5];
    if (n != 27 || !g_block.residual_norm_backward || !is_dense(a[18], &dx) || dx.last <= 0 || dx.last > 8192 || !alike(a[0], &dx, -1, &dz) ||
        !alike(a[1], &dx, dx.type, &dxo) || !alike(a[2], &dx, dx.type, &xo) || !alike(a[3], &dx, -1, &h) || !alike(a[19], &dx, h.type, &dh))
        GENERAL;
    /* a gradient that is to be made: of h, the gate and the four parameters */
    static const int of[6] = {3, 5, 7, 8, 10, 11};
    for (int i = 0; i < 6; ++i)
        if ((a[of[i]] == Py_None) != (a[19 + i] == Py_None)) GENERAL;
    const int64_t rows = dx.count / dx.last, cols = dx.last;
    if (!residual(a + 5, a + 14, rows, cols, &r) || !vector(a[4], F32, rows * 4, 0, &stats) || !vector(a[20], F32, r.gates * cols, 1, &g[0])) GENERAL;
    for (int i = 1; i < 5; ++i)
        if (!vector(a[20 + i], F32, cols, 1, &g[i])) GENERAL;
    r.eps = 1.f;
    PyObject *held;
    const int ok = workspace(a[25], a[25] == Py_None ? g_block.residual_norm_backward_bytes(rows, (int)cols, r.gates) : 0, a[26], a[18], &ws, &held);
    if (ok < 0) return NULL;
    if (!ok) {
        Py_XDECREF(held);
        GENERAL;
    }
    CALL_WITH(held, g_block.residual_norm_backward(&r, dz.ptr, dz.type, cols, dxo.ptr, cols, xo.ptr, dx.type, cols, h.ptr, h.type, cols, stats, dx.ptr, cols, dh.ptr,
                                        cols, g[0], g[1], g[2], g[3], g[4], ws.ptr, bytes_of(&ws)));
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    {"bind", bind, METH_O, "bind(address of gspc_conv2d_grouped)"},
    {"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, "one grouped convolution"},
    FAST(bind_tokens), FAST(pack), FAST(unpack), FAST(quantize), FAST(dequantize), FAST(norm), FAST(norm_backward), FAST(matmul),
    FAST(bind_block), FAST(quantize_f8), FAST(dequantize_f8), FAST(matmul_f8), FAST(dropout), FAST(residual_norm), FAST(residual_norm_backward),
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gspc_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__gspc_call(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_value = PyUnicode_InternFromString("value");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_shape = PyUnicode_InternFromString("shape");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    return s_data_ptr && s_value && s_is_cuda && s_dtype && s_shape && s_is_contiguous ? PyModule_Create(&module) : NULL;
}
