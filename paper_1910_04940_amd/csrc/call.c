/* Calls from Python: what binding.py and operators.py would do with ctypes, in the usual case.
 *
 * A collective: a list of
 * tensors and plain integers.  A small payload takes the GPU 2 to 4 us and the C call 3; marshalling eight
 * tensors through ctypes took 1.1 us more (calls one after the other, 8 ranks x 16 KiB 4.6 us, 3.5 like this).
 *
 *   call(function, bufs, n_elems, dtype, schedule, stream[, redop]) -> status, or None where an argument is of
 *   another kind: the caller then goes through ctypes, which takes them all and reports what it does not take.
 *
 * An operator on tensors: reading their types, sizes and strides in Python and marshalling a dozen arguments took 4 us of a call
 * (one row of a table 6.2 us like that, 4.0 here).  Each function takes the operator's address, the dict of the types seen so far
 * (a tensor's dtype -> its code) and the operator's arguments in the order of operators.py; None where one is not as usual.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/blink.h"

typedef blink_status_t (*plain_fn)(void* const*, int, size_t, blink_dtype_t, blink_schedule_t*, void*);
typedef blink_status_t (*redop_fn)(void* const*, int, size_t, blink_dtype_t, blink_redop_t, blink_schedule_t*, void*);

static PyObject *data_ptr_name, *address_name;

/* A non-negative int of at most 64 bits; 0 if it is something else. */
static int word(PyObject* o, unsigned long long* out) {
    if (!PyLong_CheckExact(o)) return 0;
    *out = PyLong_AsUnsignedLongLong(o);
    if (*out == (unsigned long long)-1 && PyErr_Occurred()) {
        PyErr_Clear();
        return 0;
    }
    return 1;
}

static PyObject* call(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    void* bufs[BLINK_MAX_RANKS];
    unsigned long long fn, n, dtype, schedule, stream, redop = 0;
    (void)self;
    if (nargs < 6 || nargs > 7) {
        PyErr_SetString(PyExc_TypeError, "call takes 6 or 7 arguments");
        return NULL;
    }
    PyObject* const list = args[1];
    const int is_list = PyList_CheckExact(list);
    if (!(is_list || PyTuple_CheckExact(list)) || !word(args[0], &fn) || fn == 0 || !word(args[2], &n) || !word(args[3], &dtype) ||
        dtype > 0x7fffffff || !word(args[5], &stream) || (nargs == 7 && (!word(args[6], &redop) || redop > 0x7fffffff)))
        Py_RETURN_NONE;
    const Py_ssize_t k = Py_SIZE(list);
    if (k > BLINK_MAX_RANKS) Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < k; ++i) {
        if (Py_SIZE(list) != k) Py_RETURN_NONE; /* (data_ptr may be anybody's code) */
        PyObject* const b = is_list ? PyList_GET_ITEM(list, i) : PyTuple_GET_ITEM(list, i);
        unsigned long long at;
        Py_INCREF(b);
        PyObject* const p = PyLong_CheckExact(b) ? Py_NewRef(b) : PyObject_CallMethodNoArgs(b, data_ptr_name);
        Py_DECREF(b);
        if (!p) {
            if (!PyErr_ExceptionMatches(PyExc_AttributeError) && !PyErr_ExceptionMatches(PyExc_TypeError)) return NULL;
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        const int ok = word(p, &at);
        Py_DECREF(p);
        if (!ok) Py_RETURN_NONE;
        bufs[i] = (void*)at;
    }
    PyObject* const handle = PyObject_GetAttr(args[4], address_name);
    if (!handle) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const int ok = word(handle, &schedule);
    Py_DECREF(handle);
    if (!ok) Py_RETURN_NONE;
    blink_status_t status;
    Py_BEGIN_ALLOW_THREADS /* as ctypes does: a call may wait (a schedule's first one, a timed choice) */
    if (nargs == 7)
        status = ((redop_fn)fn)(bufs, (int)k, (size_t)n, (blink_dtype_t)dtype, (blink_redop_t)redop, (blink_schedule_t*)schedule,
                                (void*)stream);
    else
        status = ((plain_fn)fn)(bufs, (int)k, (size_t)n, (blink_dtype_t)dtype, (blink_schedule_t*)schedule, (void*)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)status);
}

/* ---- operators ------------------------------------------------------------------------------------------------------------ */
static PyObject *dtype_name, *cuda_name, *shape_name, *stride_name, *contiguous_name, *numel_name, *nbytes_name;

/* The usual case fails: no exception is left, and the caller goes the long way. */
static int unusual(void) {
    PyErr_Clear();
    return 0;
}
static int attribute_is_true(PyObject* t, PyObject* name, int call) {
    PyObject* const v = call ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
    if (!v) return unusual();
    const int yes = v == Py_True;
    Py_DECREF(v);
    return yes;
}
static int word_of(PyObject* o, unsigned long long* out) {   /* (o is given up) */
    if (!o) return unusual();
    const int ok = word(o, out);
    Py_DECREF(o);
    return ok;
}
/* A tensor's address and type, if it is on the GPU. */
static int tensor(PyObject* types, PyObject* t, void** at, long* code) {
    PyObject* const dtype = PyObject_GetAttr(t, dtype_name);
    if (!dtype) return unusual();
    PyObject* const known = PyDict_GetItemWithError(types, dtype);
    Py_DECREF(dtype);
    if (!known) return unusual();
    *code = PyLong_AsLong(known);
    if (*code == -1 && PyErr_Occurred()) return unusual();
    if (!attribute_is_true(t, cuda_name, 0)) return 0;
    unsigned long long w = 0;
    const int ok = word_of(PyObject_CallMethodNoArgs(t, data_ptr_name), &w);
    *at = (void*)w;
    return ok;
}
static int pair_of(PyObject* tuple, Py_ssize_t* a, Py_ssize_t* b) {
    int ok = 0;
    if (tuple && PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 2) {
        *a = PyLong_AsSsize_t(PyTuple_GET_ITEM(tuple, 0));
        *b = PyLong_AsSsize_t(PyTuple_GET_ITEM(tuple, 1));
        ok = !PyErr_Occurred() && *a >= 0 && *b >= 0;
    }
    Py_XDECREF(tuple);
    return ok ? 1 : unusual();
}
/* A matrix whose rows are contiguous. */
typedef struct {
    void* at;
    long code;
    Py_ssize_t rows, cols, stride;
} matrix_t;
static int matrix(PyObject* types, PyObject* t, matrix_t* m) {
    Py_ssize_t one;
    if (!tensor(types, t, &m->at, &m->code) || !pair_of(PyObject_GetAttr(t, shape_name), &m->rows, &m->cols) ||
        !pair_of(PyObject_CallMethodNoArgs(t, stride_name), &m->stride, &one) || (m->cols > 1 && one != 1))
        return 0;
    if (m->rows <= 1 && m->stride < m->cols) m->stride = m->cols;
    return 1;
}
static int is_float(long code) { return code == BLINK_FP32 || code == BLINK_BF16 || code == BLINK_FP16; }
/* A contiguous tensor of any shape (tokens) of `elements` (any number: -1, which is then set), of one of two types. */
static int any_shape(PyObject* types, PyObject* t, long code, long or_code, Py_ssize_t* elements, void** at, long* is) {
    long c;
    if (!tensor(types, t, at, &c) || (c != code && c != or_code) || !attribute_is_true(t, contiguous_name, 1)) return 0;
    PyObject* const n = PyObject_CallMethodNoArgs(t, numel_name);
    if (!n) return unusual();
    const Py_ssize_t many = PyLong_AsSsize_t(n);
    Py_DECREF(n);
    if (many < 0) return unusual();
    if (*elements >= 0 && many != *elements) return 0;
    *elements = many;
    *is = c;
    return 1;
}
/* The same of one type and one dimension. */
static int whole(PyObject* types, PyObject* t, long code, Py_ssize_t* elements, void** at) {
    long is;
    PyObject* const shape = PyObject_GetAttr(t, shape_name);
    if (!shape) return unusual();
    const int line = PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) == 1;
    Py_DECREF(shape);
    return line && any_shape(types, t, code, code, elements, at, &is);
}
/* Of two dimensions. */
static int table(PyObject* types, PyObject* t, long code, Py_ssize_t rows, Py_ssize_t cols, void** at) {
    Py_ssize_t r, c, n = rows * cols;
    long is;
    return pair_of(PyObject_GetAttr(t, shape_name), &r, &c) && r == rows && c == cols && any_shape(types, t, code, code, &n, at, &is);
}
static int space(PyObject* t, void** at, Py_ssize_t* bytes) {   /* a contiguous tensor of any type, or none */
    unsigned long long p = 0, n = 0;
    if (t != Py_None && !(attribute_is_true(t, cuda_name, 0) && attribute_is_true(t, contiguous_name, 1) &&
                          word_of(PyObject_CallMethodNoArgs(t, data_ptr_name), &p) && word_of(PyObject_GetAttr(t, nbytes_name), &n)))
        return 0;
    *at = (void*)p;
    *bytes = (Py_ssize_t)n;
    return 1;
}
static int number(PyObject* o, float* out) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return 0;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return unusual();
    *out = (float)v;
    return 1;
}
static int truth(PyObject* o, int* out) {
    *out = o == Py_True;
    return o == Py_True || o == Py_False;
}
static int small(PyObject* o, int* out) {
    unsigned long long w;
    if (!word(o, &w) || w > 0x7fffffff) return 0;
    *out = (int)w;
    return 1;
}
#define USUAL(condition) if (!(condition)) Py_RETURN_NONE
#define TAKES(n)                                                          \
    if (nargs != (n) || !PyDict_CheckExact(args[1])) Py_RETURN_NONE;      \
    PyObject* const types = args[1];                                      \
    unsigned long long fn, stream;                                        \
    (void)self;                                                           \
    USUAL(word(args[0], &fn) && fn != 0 && word(args[(n) - 1], &stream))
#define RUN(call)                          \
    blink_status_t status;                 \
    Py_BEGIN_ALLOW_THREADS status = call;  \
    Py_END_ALLOW_THREADS return PyLong_FromLong((long)status)

/* table, tokens, out, scale, stream */
static PyObject* embedding(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    TAKES(7);
    matrix_t t, o;
    Py_ssize_t n = -1;
    void* tokens;
    long token;
    float scale;
    USUAL(matrix(types, args[2], &t) && any_shape(types, args[3], BLINK_INT64, BLINK_INT32, &n, &tokens, &token) && matrix(types, args[4], &o) &&
          o.rows == n && o.cols == t.cols && number(args[5], &scale) && is_float(t.code) && is_float(o.code));
    RUN(((__typeof__(&blink_embedding))fn)(t.at, (blink_dtype_t)t.code, (size_t)t.rows, (size_t)t.cols, (size_t)t.stride, tokens, (blink_dtype_t)token,
                                           (size_t)n, scale, o.at, (blink_dtype_t)o.code, (size_t)o.stride, (void*)stream));
}

/* tokens, grad_out, grad_table, workspace, scale, accumulate, stream */
static PyObject* embedding_gradient(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    TAKES(9);
    matrix_t g, t;
    Py_ssize_t n = -1, size;
    void *tokens, *work;
    long token;
    float scale;
    int accumulate;
    USUAL(any_shape(types, args[2], BLINK_INT64, BLINK_INT32, &n, &tokens, &token) && matrix(types, args[3], &g) && matrix(types, args[4], &t) && g.rows == n &&
          g.cols == t.cols && space(args[5], &work, &size) && number(args[6], &scale) && truth(args[7], &accumulate) && is_float(t.code) && is_float(g.code));
    RUN(((__typeof__(&blink_embedding_gradient))fn)(tokens, (blink_dtype_t)token, (size_t)n, g.at, (blink_dtype_t)g.code, (size_t)g.stride, scale, accumulate,
                                                    t.at, (blink_dtype_t)t.code, (size_t)t.rows, (size_t)t.cols, (size_t)t.stride, work, (size_t)size,
                                                    (void*)stream));
}

/* logits, k, chosen, weights, counts, sums, workspace, keep, normalize, stream */
static PyObject* route(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    TAKES(12);
    matrix_t x;
    Py_ssize_t size, n, e;
    void *chosen, *weights, *counts, *sums, *work, *keep = NULL;
    int k, normalize;
    USUAL(matrix(types, args[2], &x) && is_float(x.code) && x.cols < 0x7fffffff && small(args[3], &k));
    n = x.rows;
    e = x.cols + 1;
    USUAL(table(types, args[4], BLINK_INT32, n, k, &chosen) && table(types, args[5], BLINK_FP32, n, k, &weights) &&
          whole(types, args[6], BLINK_INT32, &e, &counts) && whole(types, args[7], BLINK_FP32, &e, &sums) &&
          space(args[8], &work, &size) && (args[9] == Py_None || whole(types, args[9], -1, &n, &keep)) && truth(args[10], &normalize));
    RUN(((__typeof__(&blink_route))fn)(x.at, (blink_dtype_t)x.code, (size_t)x.rows, (int)x.cols, (size_t)x.stride, keep, k, normalize, chosen, weights, counts,
                                       sums, work, (size_t)size, (void*)stream));
}

/* counts, sums, k, loss, balance, z, stream */
static PyObject* route_loss(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    TAKES(9);
    Py_ssize_t e = -1, three = 3;
    void *counts, *sums, *loss;
    int k;
    float balance, z;
    USUAL(whole(types, args[2], BLINK_INT32, &e, &counts) && e > 0 && e <= 0x7fffffff &&
          whole(types, args[3], BLINK_FP32, &e, &sums) && small(args[4], &k) &&
          whole(types, args[5], BLINK_FP32, &three, &loss) && number(args[6], &balance) && number(args[7], &z));
    RUN(((__typeof__(&blink_route_loss))fn)(counts, sums, (int)(e - 1), k, balance, z, loss, (void*)stream));
}

/* logits, k, chosen, counts, grad_logits, keep, normalize, grad_weights, grad_loss, balance, z, stream */
static PyObject* route_gradient(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
    TAKES(14);
    matrix_t x, g;
    Py_ssize_t n, e, one = 1;
    void *chosen, *counts, *keep = NULL, *by_weight = NULL, *up = NULL;
    int k, normalize;
    float balance, z;
    USUAL(matrix(types, args[2], &x) && is_float(x.code) && x.cols < 0x7fffffff && small(args[3], &k) && matrix(types, args[6], &g) && g.code == x.code &&
          g.rows == x.rows && g.cols == x.cols);
    n = x.rows;
    e = x.cols + 1;
    USUAL(table(types, args[4], BLINK_INT32, n, k, &chosen) && whole(types, args[5], BLINK_INT32, &e, &counts) &&
          (args[7] == Py_None || whole(types, args[7], -1, &n, &keep)) && truth(args[8], &normalize) &&
          (args[9] == Py_None || table(types, args[9], BLINK_FP32, n, k, &by_weight)) &&
          (args[10] == Py_None || whole(types, args[10], BLINK_FP32, &one, &up)) && number(args[11], &balance) && number(args[12], &z));
    RUN(((__typeof__(&blink_route_gradient))fn)(x.at, (blink_dtype_t)x.code, (size_t)x.rows, (int)x.cols, (size_t)x.stride, keep, k, normalize, chosen, by_weight,
                                                counts, up, balance, z, g.at, (size_t)g.stride, (void*)stream));
}

static PyMethodDef methods[] = {
    {"call", (PyCFunction)(void (*)(void))call, METH_FASTCALL, NULL},
    {"embedding", (PyCFunction)(void (*)(void))embedding, METH_FASTCALL, NULL},
    {"embedding_gradient", (PyCFunction)(void (*)(void))embedding_gradient, METH_FASTCALL, NULL},
    {"route", (PyCFunction)(void (*)(void))route, METH_FASTCALL, NULL},
    {"route_loss", (PyCFunction)(void (*)(void))route_loss, METH_FASTCALL, NULL},
    {"route_gradient", (PyCFunction)(void (*)(void))route_gradient, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_blinkcall", NULL, 0, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__blinkcall(void) {
    data_ptr_name = PyUnicode_InternFromString("data_ptr");
    address_name = PyUnicode_InternFromString("_address");
    dtype_name = PyUnicode_InternFromString("dtype");
    cuda_name = PyUnicode_InternFromString("is_cuda");
    shape_name = PyUnicode_InternFromString("shape");
    stride_name = PyUnicode_InternFromString("stride");
    contiguous_name = PyUnicode_InternFromString("is_contiguous");
    numel_name = PyUnicode_InternFromString("numel");
    nbytes_name = PyUnicode_InternFromString("nbytes");
    if (!data_ptr_name || !address_name || !dtype_name || !cuda_name || !shape_name || !stride_name || !contiguous_name || !numel_name || !nbytes_name) return NULL;
    return PyModule_Create(&module);
}
