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
static PyObject *g_types[3];               /* torch.float32, bfloat16, int8, in the order of the library's numbers */
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

/* A contiguous tensor on the GPU of one of the three types.  0: not one (no exception is left). */
static int tensor(PyObject *t, tensor_t *o) {
    if (!is_true(PyObject_GetAttr(t, s_is_cuda))) goto no;
    PyObject *v = PyObject_GetAttr(t, s_dtype);
    if (!v) goto no;
    for (o->type = 0; o->type < 3 && v != g_types[o->type]; ++o->type) {}
    Py_DECREF(v);
    if (o->type == 3 || !is_true(PyObject_CallMethodNoArgs(t, s_is_contiguous))) goto no;
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
/* One of a type and of a number of elements, or NULL where none is allowed. */
static int vector(PyObject *t, int type, int64_t count, int none, void **ptr) {
    tensor_t o;
    *ptr = NULL;
    if (t == Py_None) return none;
    if (!tensor(t, &o) || o.type != type || o.count != count) return 0;
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

static size_t bytes_of(const tensor_t *t) { return t->ptr ? (size_t)t->count * (t->type == 0 ? 4 : t->type == 1 ? 2 : 1) : 0; }

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

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    {"bind", bind, METH_O, "bind(address of gspc_conv2d_grouped)"},
    {"conv", (PyCFunction)(void (*)(void))conv, METH_FASTCALL, "one grouped convolution"},
    FAST(bind_tokens), FAST(pack), FAST(unpack), FAST(quantize), FAST(dequantize), FAST(norm), FAST(norm_backward), FAST(matmul),
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
