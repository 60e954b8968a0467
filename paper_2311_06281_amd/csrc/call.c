/* The scan's and the operators' entry points as Python calls: arguments taken as they are and handed to the library.
 *
 * The smallest calls are bound by the host.  ctypes takes about 0.5 us to convert ten arguments and a Python frame
 * with the four data_ptr() calls another 0.5, beside 3.1 us for the launch itself; here it is 0.4 together.  An
 * operator has about twice the arguments: a norm of 64 rows takes 6.0 us through ctypes, the launch included, and 3.9 this way. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef int (*scan_fn)(const void *, const void *, const void *, void *, int64_t, int64_t, int64_t, int, uint32_t, void *);

static scan_fn entry[2]; /* heinsen_scan, heinsen_scan_static */
static PyObject *name_data_ptr, *name_cuda_stream;

/* What `x`, a Python integer, holds, reduced to 64 bits as ctypes does it.  0: it is no integer. */
static int integer(PyObject *x, uint64_t *v)
{
    if (!PyLong_Check(x)) return 0;
    *v = PyLong_AsUnsignedLongLongMask(x);
    return 1;
}

/* Address behind `x`: None, an integer, or what its method or attribute `name` gives.  0: none of these (an exception
 * is set unless there is merely no integer). */
static int address(PyObject *x, PyObject *name, int is_method, uint64_t *v)
{
    if (x == Py_None) {
        *v = 0;
        return 1;
    }
    if (PyLong_CheckExact(x)) return integer(x, v);
    PyObject *r = is_method ? PyObject_CallMethodNoArgs(x, name) : PyObject_GetAttr(x, name);
    if (r == NULL) return 0;
    const int ok = integer(r, v);
    Py_DECREF(r);
    return ok;
}

/* (a, b, x0, out, B, D, n, layout, flags, stream) -> status, or NotImplemented where some argument is of another kind
 * than these (the caller then converts them one by one, which also says what is wrong). */
static PyObject *call(int which, PyObject *const *args, Py_ssize_t nargs)
{
    uint64_t p[4], v[5], stream;
    if (nargs != 10 || entry[which] == NULL) Py_RETURN_NOTIMPLEMENTED;
    /* where the caller deals in addresses and handles, its numbers are looked at before any tensor is asked for its own */
    if (PyLong_CheckExact(args[0]) || PyLong_CheckExact(args[9]) || args[9] == Py_None)
        for (int i = 0; i < 5; ++i)
            if (!PyLong_Check(args[4 + i])) goto other;
    for (int i = 0; i < 4; ++i)
        if (!address(args[i], name_data_ptr, 1, &p[i])) goto other;
    for (int i = 0; i < 5; ++i)
        if (!integer(args[4 + i], &v[i])) goto other;
    if (!address(args[9], name_cuda_stream, 0, &stream)) goto other;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = entry[which]((const void *)(uintptr_t)p[0], (const void *)(uintptr_t)p[1], (const void *)(uintptr_t)p[2], (void *)(uintptr_t)p[3],
                          (int64_t)v[0], (int64_t)v[1], (int64_t)v[2], (int)v[3], (uint32_t)v[4], (void *)(uintptr_t)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
other:
    if (PyErr_Occurred()) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError) && !PyErr_ExceptionMatches(PyExc_TypeError)) return NULL;
        PyErr_Clear();
    }
    Py_RETURN_NOTIMPLEMENTED;
}

static PyObject *scan(PyObject *self, PyObject *const *args, Py_ssize_t nargs) { return call(0, args, nargs); }
static PyObject *scan_static(PyObject *self, PyObject *const *args, Py_ssize_t nargs) { return call(1, args, nargs); }

/* The operators: pointers, 64-bit integers, a float32, flags and a stream, in the order of the library's arguments. */
enum { ATTENTION, ATTENTION_BACKWARD, NORM, NORM_BACKWARD, OPERATORS };
static const int pointers_of[OPERATORS] = {8, 13, 8, 14}, integers_of[OPERATORS] = {9, 9, 4, 4};
static void (*operators[OPERATORS])(void);

#define P const void *
#define I int64_t
typedef int (*attention_fn)(P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, I, float, uint32_t, void *);
typedef int (*attention_backward_fn)(P, P, P, P, P, P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, I, I, float, uint32_t, void *);
typedef int (*norm_fn)(P, P, P, P, P, P, P, P, I, I, I, I, float, uint32_t, void *);
typedef int (*norm_backward_fn)(P, P, P, P, P, P, P, P, P, P, P, P, P, P, I, I, I, I, float, uint32_t, void *);
#undef P
#undef I

/* As call(): status, or NotImplemented. */
static PyObject *call_operator(int which, PyObject *const *args, Py_ssize_t nargs)
{
    const int np = pointers_of[which], ni = integers_of[which];
    uint64_t address_of[14], v[9], flags, stream;
    const void *p[14];
    int64_t i[9];
    if (nargs != np + ni + 3 || operators[which] == NULL) Py_RETURN_NOTIMPLEMENTED;
    PyObject *const *const rest = args + np + ni;
    /* numbers first: no tensor is asked for its address in vain */
    for (int k = 0; k < ni; ++k)
        if (!integer(args[np + k], &v[k])) goto other;
    if (!PyFloat_Check(rest[0]) || !integer(rest[1], &flags)) goto other;
    for (int k = 0; k < np; ++k)
        if (!address(args[k], name_data_ptr, 1, &address_of[k])) goto other;
    if (!address(rest[2], name_cuda_stream, 0, &stream)) goto other;
    const float x = (float)PyFloat_AS_DOUBLE(rest[0]);
    const uint32_t f = (uint32_t)flags;
    void *const s = (void *)(uintptr_t)stream;
    for (int k = 0; k < np; ++k) p[k] = (const void *)(uintptr_t)address_of[k];
    for (int k = 0; k < ni; ++k) i[k] = (int64_t)v[k];
    int status;
    Py_BEGIN_ALLOW_THREADS
    switch (which) {
    case ATTENTION:
        status = ((attention_fn)operators[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], i[0], i[1], i[2], i[3], i[4], i[5], i[6], i[7],
                                                  i[8], x, f, s);
        break;
    case ATTENTION_BACKWARD:
        status = ((attention_backward_fn)operators[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], i[0],
                                                           i[1], i[2], i[3], i[4], i[5], i[6], i[7], i[8], x, f, s);
        break;
    case NORM:
        status = ((norm_fn)operators[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], i[0], i[1], i[2], i[3], x, f, s);
        break;
    default:
        status = ((norm_backward_fn)operators[which])(p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9], p[10], p[11], p[12], p[13], i[0],
                                                      i[1], i[2], i[3], x, f, s);
    }
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
other:
    if (PyErr_Occurred()) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError) && !PyErr_ExceptionMatches(PyExc_TypeError)) return NULL;
        PyErr_Clear();
    }
    Py_RETURN_NOTIMPLEMENTED;
}

static PyObject *linear_attention(PyObject *self, PyObject *const *args, Py_ssize_t nargs) { return call_operator(ATTENTION, args, nargs); }
static PyObject *linear_attention_backward(PyObject *self, PyObject *const *args, Py_ssize_t nargs)
{
    return call_operator(ATTENTION_BACKWARD, args, nargs);
}
static PyObject *block_norm(PyObject *self, PyObject *const *args, Py_ssize_t nargs) { return call_operator(NORM, args, nargs); }
static PyObject *block_norm_backward(PyObject *self, PyObject *const *args, Py_ssize_t nargs) { return call_operator(NORM_BACKWARD, args, nargs); }

/* bind_operators(the addresses of the four entry points in the order above) */
static PyObject *bind_operators(PyObject *self, PyObject *args)
{
    unsigned long long f[OPERATORS];
    if (!PyArg_ParseTuple(args, "KKKK", &f[0], &f[1], &f[2], &f[3])) return NULL;
    for (int k = 0; k < OPERATORS; ++k) operators[k] = (void (*)(void))(uintptr_t)f[k];
    Py_RETURN_NONE;
}

/* bind(address of heinsen_scan, address of heinsen_scan_static) */
static PyObject *bind(PyObject *self, PyObject *args)
{
    unsigned long long f, g;
    if (!PyArg_ParseTuple(args, "KK", &f, &g)) return NULL;
    entry[0] = (scan_fn)(uintptr_t)f;
    entry[1] = (scan_fn)(uintptr_t)g;
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {
    {"scan", (PyCFunction)(void (*)(void))scan, METH_FASTCALL, NULL},
    {"scan_static", (PyCFunction)(void (*)(void))scan_static, METH_FASTCALL, NULL},
    {"bind", bind, METH_VARARGS, NULL},
    {"linear_attention", (PyCFunction)(void (*)(void))linear_attention, METH_FASTCALL, NULL},
    {"linear_attention_backward", (PyCFunction)(void (*)(void))linear_attention_backward, METH_FASTCALL, NULL},
    {"block_norm", (PyCFunction)(void (*)(void))block_norm, METH_FASTCALL, NULL},
    {"block_norm_backward", (PyCFunction)(void (*)(void))block_norm_backward, METH_FASTCALL, NULL},
    {"bind_operators", bind_operators, METH_VARARGS, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__call(void)
{
    name_data_ptr = PyUnicode_InternFromString("data_ptr");
    name_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (name_data_ptr == NULL || name_cuda_stream == NULL) return NULL;
    return PyModule_Create(&module);
}
