/*
 * The usual case of the operators' calls from Python, in C: torch tensors to pointers, row lengths and types.
 *
 * A call of an operator from Python is half of what the smallest ones cost (a norm of one row: 8 us with its 3 us kernel), and
 * that is mostly attributes of tensors being read one by one.  Each function here reads them and calls the library where
 * every operand is as expected, and returns the library's code; where one is not, it returns None without having called, and
 * binding.py's own checks say what is wrong, or take what is unusual but right.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/reft.h"

enum { FLOATS = 1 << REFT_F32 | 1 << REFT_BF16 | 1 << REFT_F16, EIGHTS = 1 << REFT_E4M3 | 1 << REFT_E5M2 };

static PyObject *s_dtype, *s_shape, *s_stride, *s_data_ptr, *s_stream, *s_size, *s_device;
static int here;                               /* the current GPU in the call under way (all calls hold the interpreter's lock) */

int hipGetDevice(int *device);                 /* of the HIP runtime that the library is linked with; 0: success */
static PyObject *known[5];                     /* torch's dtypes by the library's numbers, as they have been met */

typedef struct {
    void *p;
    uint64_t ld, n[3], step[3];
    int type;
} operand;

/* A sequence of `count` whole numbers.  All functions: 1 if so, 0 if not (no error is left set). */
static int numbers(PyObject *t, int count, uint64_t *out)
{
    int ok = t && PyTuple_Check(t) && PyTuple_GET_SIZE(t) == count;
    for (int i = 0; ok && i < count; ++i) {
        const long long v = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
        ok = v >= 0 && !PyErr_Occurred();
        out[i] = (uint64_t)v;
    }
    Py_XDECREF(t);
    PyErr_Clear();
    return ok;
}

static int type_of(PyObject *t, int *type)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    *type = -1;
    for (int i = 0; i < 5 && d; ++i)
        if (d == known[i]) *type = i;
    Py_XDECREF(d);
    PyErr_Clear();
    return *type >= 0;
}

/* A call of `want` arguments begins. */
static int begin(Py_ssize_t n, Py_ssize_t want)
{
    if (hipGetDevice(&here)) here = -2;
    return n == want;
}

/* The tensor is memory of the current GPU (of none: -1). */
static int seen(PyObject *t)
{
    PyObject *d = PyObject_CallMethodNoArgs(t, s_device);
    const int ok = d && here >= 0 && PyLong_AsLong(d) == here;
    Py_XDECREF(d);
    PyErr_Clear();
    return ok;
}

static int address_of(PyObject *t, void **p)
{
    if (!seen(t)) return 0;
    PyObject *a = PyObject_CallMethodNoArgs(t, s_data_ptr);
    *p = a ? PyLong_AsVoidPtr(a) : NULL;
    Py_XDECREF(a);
    const int ok = !PyErr_Occurred();
    PyErr_Clear();
    return ok;
}

/* A matrix with contiguous rows of one of `types`; of another's shape where `like` is given.  None: left out, if it may be. */
static int matrix(PyObject *t, int optional, const uint64_t *like, int types, operand *o)
{
    o->p = NULL, o->ld = 0, o->type = -1;
    if (t == Py_None) return optional;
    return numbers(PyObject_GetAttr(t, s_shape), 2, o->n) && (!like || (o->n[0] == like[0] && o->n[1] == like[1])) &&
           numbers(PyObject_CallMethodNoArgs(t, s_stride), 2, o->step) && o->step[1] == 1 && o->step[0] >= o->n[1] &&
           type_of(t, &o->type) && (types >> o->type & 1) && address_of(t, &o->p) && (o->ld = o->step[0], 1);
}

static int vector(PyObject *t, int optional, uint64_t n, int types, operand *o)
{
    o->p = NULL, o->type = -1;
    if (t == Py_None) return optional;
    return numbers(PyObject_GetAttr(t, s_shape), 1, o->n) && o->n[0] == n && numbers(PyObject_CallMethodNoArgs(t, s_stride), 1, o->step) &&
           o->step[0] == 1 && type_of(t, &o->type) && (types >> o->type & 1) && address_of(t, &o->p);
}

/* Scales: bytes [ceil(cols / 512)][rows][4], without gaps. */
static int scales(PyObject *t, int optional, uint64_t rows, uint64_t cols, operand *o)
{
    o->p = NULL, o->ld = 0;
    if (t == Py_None) return optional;
    uint64_t size = 0;
    PyObject *one = PyObject_GetAttr(t, s_size);             /* itemsize */
    if (one) size = PyLong_AsUnsignedLongLong(one);
    Py_XDECREF(one);
    PyErr_Clear();
    return size == 1 && numbers(PyObject_GetAttr(t, s_shape), 3, o->n) && o->n[0] == (cols + 511) / 512 && o->n[1] == rows && o->n[2] == 4 &&
           numbers(PyObject_CallMethodNoArgs(t, s_stride), 3, o->step) && o->step[2] == 1 && o->step[1] == 4 && (o->step[0] == 4 * rows || !rows) &&
           address_of(t, &o->p) && (o->ld = rows, 1);
}

/* Scratch memory: a contiguous vector of bytes. */
static int scratch(PyObject *t, operand *o)
{
    o->p = NULL, o->n[0] = 0;
    if (t == Py_None) return 1;
    uint64_t size = 0;
    PyObject *one = PyObject_GetAttr(t, s_size);
    if (one) size = PyLong_AsUnsignedLongLong(one);
    Py_XDECREF(one);
    PyErr_Clear();
    return size == 1 && numbers(PyObject_GetAttr(t, s_shape), 1, o->n) && numbers(PyObject_CallMethodNoArgs(t, s_stride), 1, o->step) &&
           (o->step[0] == 1 || o->n[0] <= 1) && address_of(t, &o->p);
}

/* None, a number or torch's stream. */
static int stream_of(PyObject *s, void **out)
{
    *out = NULL;
    if (s == Py_None) return 1;
    if (PyLong_Check(s)) {
        *out = PyLong_AsVoidPtr(s);
    } else {
        PyObject *a = PyObject_GetAttr(s, s_stream);
        if (!a) return PyErr_Clear(), 0;
        *out = PyLong_AsVoidPtr(a);
        Py_DECREF(a);
    }
    const int ok = !PyErr_Occurred();
    PyErr_Clear();
    return ok;
}

static int real(PyObject *v, double *out)
{
    *out = PyFloat_AsDouble(v);
    const int ok = !PyErr_Occurred();
    PyErr_Clear();
    return ok;
}

static int whole(PyObject *v, uint64_t *out)
{
    *out = PyLong_Check(v) ? PyLong_AsUnsignedLongLong(v) : 0;
    const int ok = PyLong_Check(v) && !PyErr_Occurred();
    PyErr_Clear();
    return ok;
}

#define OTHERWISE(cond) if (!(cond)) Py_RETURN_NONE
#define CALL(expr)                                                                                \
    do {                                                                                          \
        int rc;                                                                                   \
        Py_BEGIN_ALLOW_THREADS rc = (expr);                                                       \
        Py_END_ALLOW_THREADS return PyLong_FromLong(rc);                                          \
    } while (0)

static int or_f32(int type) { return 1 << type | 1 << REFT_F32; }

static PyObject *py_dropout(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    operand x, y;
    double p;
    uint64_t seed, offset;
    void *stream;
    OTHERWISE(begin(n, 6) && matrix(v[0], 0, NULL, FLOATS, &x) && matrix(v[1], 0, x.n, 1 << x.type, &y) && real(v[2], &p) && whole(v[3], &seed) &&
              whole(v[4], &offset) && stream_of(v[5], &stream));
    CALL(reft_dropout(x.p, x.ld, y.p, y.ld, x.n[0], x.n[1], x.type, p, seed, offset, stream));
}

static PyObject *py_norm_forward(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    operand x, r, w, h, rstd, y, q, s;
    double eps, p;
    uint64_t seed, offset;
    void *stream;
    OTHERWISE(begin(n, 13) && matrix(v[0], 0, NULL, FLOATS, &x) && matrix(v[1], 1, x.n, or_f32(x.type), &r) &&
              vector(v[2], 0, x.n[1], or_f32(x.type), &w) && real(v[3], &eps) && real(v[4], &p) && whole(v[5], &seed) && whole(v[6], &offset) &&
              matrix(v[7], 1, x.n, r.type < 0 ? or_f32(x.type) : 1 << r.type, &h) && vector(v[8], 1, x.n[0], 1 << REFT_F32, &rstd) &&
              matrix(v[9], 1, x.n, 1 << x.type, &y) && matrix(v[10], 1, x.n, EIGHTS, &q) && scales(v[11], 1, x.n[0], x.n[1], &s) &&
              stream_of(v[12], &stream));
    CALL(reft_norm_forward(x.p, x.ld, r.p, r.ld, w.p, x.n[0], x.n[1], x.type, r.type >= 0 ? r.type : h.type >= 0 ? h.type : x.type, w.type,
                           eps, p, seed, offset, h.p, h.ld, rstd.p, y.p, y.ld, q.p, q.ld, q.type, s.p, s.ld, stream));
}

static PyObject *py_norm_backward(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    operand dy, dh, h, rstd, w, dres, dx, dw, room;
    double p;
    uint64_t seed, offset;
    void *stream;
    OTHERWISE(begin(n, 13) && matrix(v[0], 0, NULL, FLOATS, &dy) && matrix(v[2], 0, dy.n, or_f32(dy.type), &h) &&
              matrix(v[1], 1, dy.n, 1 << h.type, &dh) && vector(v[3], 0, dy.n[0], 1 << REFT_F32, &rstd) &&
              vector(v[4], 0, dy.n[1], or_f32(dy.type), &w) && real(v[5], &p) && whole(v[6], &seed) && whole(v[7], &offset) &&
              matrix(v[8], 1, dy.n, 1 << h.type, &dres) && matrix(v[9], 1, dy.n, 1 << dy.type, &dx) &&
              vector(v[10], 1, dy.n[1], 1 << REFT_F32, &dw) && scratch(v[11], &room) && stream_of(v[12], &stream));
    CALL(reft_norm_backward(dy.p, dy.ld, dh.p, dh.ld, h.p, h.ld, rstd.p, w.p, dy.n[0], dy.n[1], dy.type, h.type, w.type, p, seed, offset, dres.p,
                            dres.ld, dx.p, dx.ld, dw.p, room.p, room.n[0], stream));
}

static PyObject *py_quantize(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    operand x, q, s, qt, st;
    void *stream;
    OTHERWISE(begin(n, 7) && matrix(v[0], 0, NULL, FLOATS, &x));
    const int blocks = PyObject_IsTrue(v[5]);
    const uint64_t turned[2] = {x.n[1], x.n[0]};
    PyErr_Clear();
    OTHERWISE(blocks >= 0 && matrix(v[1], 1, x.n, EIGHTS, &q) && matrix(v[3], 1, turned, q.type < 0 ? EIGHTS : 1 << q.type, &qt) &&
              scales(v[2], 1, blocks ? (x.n[0] + 127) / 128 : x.n[0], x.n[1], &s) &&
              scales(v[4], 1, blocks ? (x.n[1] + 127) / 128 : x.n[1], x.n[0], &st) && stream_of(v[6], &stream));
    CALL(reft_quantize(x.p, x.ld, x.n[0], x.n[1], x.type, q.type >= 0 ? q.type : qt.type, blocks, q.p, q.ld, s.p, s.ld, qt.p, qt.ld, st.p, st.ld,
                       stream));
}

static PyObject *py_product(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    operand a, sa, b, sb, c, room;
    void *stream;
    OTHERWISE(begin(n, 8) && matrix(v[0], 0, NULL, EIGHTS, &a) && matrix(v[2], 0, NULL, EIGHTS, &b) && a.n[1] == b.n[1]);
    const int blocks = PyObject_IsTrue(v[6]);
    const uint64_t shape[2] = {a.n[0], b.n[0]};
    PyErr_Clear();
    OTHERWISE(blocks >= 0 && scales(v[1], 1, a.n[0], a.n[1], &sa) && scales(v[3], 1, blocks ? (b.n[0] + 127) / 128 : b.n[0], b.n[1], &sb) &&
              matrix(v[4], 0, shape, FLOATS, &c) && scratch(v[5], &room) && stream_of(v[7], &stream));
    CALL(reft_product(a.p, a.ld, a.type, sa.p, sa.ld, b.p, b.ld, b.type, sb.p, sb.ld, blocks, a.n[0], b.n[0], a.n[1], c.p, c.ld, c.type, room.p,
                      room.n[0], stream));
}

/* know(dtype, number) */
static PyObject *py_know(PyObject *self, PyObject *const *v, Py_ssize_t n)
{
    const long i = n == 2 ? PyLong_AsLong(v[1]) : -1;
    if (PyErr_Occurred()) return NULL;
    if (i < 0 || i >= 5) {
        PyErr_SetString(PyExc_ValueError, "know(dtype, number of a type)");
        return NULL;
    }
    Py_INCREF(v[0]);
    Py_XSETREF(known[i], v[0]);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {METHOD(dropout), METHOD(norm_forward), METHOD(norm_backward), METHOD(quantize),
                                METHOD(product), METHOD(know), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__marshal(void)
{
    s_dtype = PyUnicode_InternFromString("dtype");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_stream = PyUnicode_InternFromString("cuda_stream");
    s_size = PyUnicode_InternFromString("itemsize");
    s_device = PyUnicode_InternFromString("get_device");
    if (!s_dtype || !s_shape || !s_stride || !s_data_ptr || !s_stream || !s_size || !s_device) return NULL;
    return PyModule_Create(&module);
}
