/* What the extension modules of the binding's operators share: strided tensors into views, flat arrays, streams and numbers from Python's objects, checked.
 * Internal to csrc/. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "sdl.h"

static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_shape, *s_stride, *s_dtype, *s_numel, *s_element_size;
static PyObject *t_float32, *t_bfloat16, *t_int32, *t_float64, *t_int64;        /* torch's types, of which a module keeps those it needs */
static PyObject *f_stream, *f_initialized, *f_device, *f_raw_stream;

typedef struct {
    sdl_view_t view;
    uint32_t shape[4];      /* batch, tokens, heads, width */
    Py_ssize_t dims;
    PyObject* dtype;        /* borrowed: one of those above, or None for another */
} Operand;

static inline int number(PyObject* v, long long* out)
{
    *out = PyLong_AsLongLong(v);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* a method without arguments that gives a number */
static inline int ask(PyObject* t, PyObject* name, long long* out)
{
    PyObject* r = PyObject_CallMethodNoArgs(t, name);
    int rc = -1;
    if (!r) return -1;
    if (name == s_data_ptr) {
        *out = (long long)PyLong_AsUnsignedLongLong(r);
        rc = PyErr_Occurred() ? -1 : 0;
    } else {
        rc = number(r, out);
    }
    Py_DECREF(r);
    return rc;
}

static inline int on_device(PyObject* t)
{
    PyObject* r = PyObject_GetAttr(t, s_is_cuda);
    int yes;
    if (!r) return -1;
    yes = PyObject_IsTrue(r);
    Py_DECREF(r);
    if (yes < 0) return -1;
    if (!yes) {
        PyErr_SetString(PyExc_ValueError, "sdl calls take device tensors; there is no CPU path");
        return -1;
    }
    return 0;
}

static inline PyObject* type_of(PyObject* t)
{
    PyObject *r = PyObject_GetAttr(t, s_dtype), *known;
    if (!r) return NULL;
    known = r == t_float32 || r == t_bfloat16 || r == t_int32 || r == t_float64 || r == t_int64 ? r : Py_None;
    Py_DECREF(r);           /* the module keeps them */
    return known;
}

static inline int dtype_number(PyObject* dtype, sdl_dtype_t* out)
{
    if (dtype == t_bfloat16) *out = SDL_DTYPE_BF16;
    else if (dtype == t_float32) *out = SDL_DTYPE_FP32;
    else {
        PyErr_SetString(PyExc_ValueError, "the operators take float32 and bfloat16");
        return -1;
    }
    return 0;
}

/* A tensor of one to four dimensions as [batch, tokens, heads, width]: what is missing is in front of the tokens, or is one head. */
static inline int operand(PyObject* t, Operand* o)
{
    static const int to[5][4] = {{0}, {3}, {1, 3}, {0, 1, 3}, {0, 1, 2, 3}};
    PyObject *shape = NULL, *stride = NULL;
    long long size, step, at, steps[4] = {0, 0, 0, 1};
    Py_ssize_t i;
    int rc = -1;
    if (on_device(t) < 0 || !(o->dtype = type_of(t)) || ask(t, s_data_ptr, &at) < 0) return -1;
    shape = PyObject_GetAttr(t, s_shape);
    stride = shape ? PyObject_CallMethodNoArgs(t, s_stride) : NULL;
    if (!stride) goto done;
    if (!PyTuple_Check(shape) || !PyTuple_Check(stride) || PyTuple_GET_SIZE(shape) != PyTuple_GET_SIZE(stride) || PyTuple_GET_SIZE(shape) < 1 ||
        PyTuple_GET_SIZE(shape) > 4) {
        PyErr_SetString(PyExc_ValueError, "the operators take tensors of one to four dimensions");
        goto done;
    }
    o->dims = PyTuple_GET_SIZE(shape);
    for (i = 0; i < 4; ++i) o->shape[i] = 1;
    for (i = 0; i < o->dims; ++i) {
        const int k = to[o->dims][i];
        if (number(PyTuple_GET_ITEM(shape, i), &size) < 0 || number(PyTuple_GET_ITEM(stride, i), &step) < 0) goto done;
        if (size < 0 || size > (long long)UINT32_MAX) {
            PyErr_SetString(PyExc_ValueError, "a dimension of 2^32 and more");
            goto done;
        }
        o->shape[k] = (uint32_t)size;
        steps[k] = step;
    }
    if (steps[3] != 1 && o->shape[3] > 1) {
        PyErr_SetString(PyExc_ValueError, "neighbouring elements of a row must be neighbours in memory");
        goto done;
    }
    o->view.data = (void*)(uintptr_t)(unsigned long long)at;
    o->view.stride_batch = steps[0];
    o->view.stride_token = steps[1];
    o->view.stride_head = steps[2];
    rc = 0;
done:
    Py_XDECREF(shape);
    Py_XDECREF(stride);
    return rc;
}

/* One whose shape and type have to be another's. */
static inline int operand_like(PyObject* t, const Operand* like, Operand* o)
{
    int i, same;
    if (operand(t, o) < 0) return -1;
    same = o->dims == like->dims;
    for (i = 0; i < 4; ++i) same = same && o->shape[i] == like->shape[i];
    if (!same) {
        PyErr_SetString(PyExc_ValueError, "a tensor of another shape than the one it belongs to");
        return -1;
    }
    if (o->dtype != like->dtype) {
        PyErr_Format(PyExc_ValueError, "a tensor of another type where %R is needed", like->dtype);
        return -1;
    }
    return 0;
}

/* Address of a contiguous array of that many elements; None is the null pointer.  dtype NULL: any. */
static inline int flat(PyObject* t, unsigned long long numel, PyObject* dtype, const char* what, void** out)
{
    PyObject* r;
    long long n, at;
    int contiguous;
    *out = NULL;
    if (t == Py_None) return 0;
    if (on_device(t) < 0) return -1;
    r = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!r) return -1;
    contiguous = PyObject_IsTrue(r);
    Py_DECREF(r);
    if (contiguous < 0) return -1;
    if (!contiguous) {
        PyErr_SetString(PyExc_ValueError, "sdl calls take contiguous tensors");
        return -1;
    }
    if (dtype) {
        if (!(r = type_of(t)) || ask(t, s_numel, &n) < 0) return -1;
        if (r != dtype || n < 0 || (unsigned long long)n != numel) {
            PyErr_Format(PyExc_ValueError, "%s: %llu elements of %R are needed", what, numel, dtype);
            return -1;
        }
    }
    if (ask(t, s_data_ptr, &at) < 0) return -1;
    *out = (void*)(uintptr_t)(unsigned long long)at;
    return 0;
}

static inline int space(PyObject* t, void** at, size_t* bytes)
{
    long long n, each;
    *bytes = 0;
    if (flat(t, 0, NULL, "workspace", at) < 0) return -1;
    if (t == Py_None) return 0;
    if (ask(t, s_numel, &n) < 0 || ask(t, s_element_size, &each) < 0) return -1;
    *bytes = (size_t)n * (size_t)each;
    return 0;
}

static inline int stream_of(PyObject* v, void** out)
{
    PyObject *r = NULL, *d;
    int ready;
    if (v == Py_None && f_raw_stream != Py_None) {
        r = PyObject_CallNoArgs(f_initialized);
        if (!r) return -1;
        ready = PyObject_IsTrue(r);
        Py_DECREF(r);
        if (ready < 0) return -1;
        if (ready) {
            d = PyObject_CallNoArgs(f_device);
            if (!d) return -1;
            r = PyObject_CallOneArg(f_raw_stream, d);
            Py_DECREF(d);
        } else {
            r = PyObject_CallOneArg(f_stream, v);
        }
    } else {
        r = PyObject_CallOneArg(f_stream, v);
    }
    if (!r) return -1;
    *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(r);
    Py_DECREF(r);
    return PyErr_Occurred() ? -1 : 0;
}

static inline int real(PyObject* v, float* out)
{
    const double x = PyFloat_AsDouble(v);
    if (x == -1.0 && PyErr_Occurred()) return -1;
    *out = (float)x;
    return 0;
}

static inline int integer(PyObject* v, int32_t* out)
{
    long long x;
    if (number(v, &x) < 0) return -1;
    if (x < INT32_MIN || x > INT32_MAX) {
        PyErr_SetString(PyExc_ValueError, "an integer of 32 bits is needed");
        return -1;
    }
    *out = (int32_t)x;
    return 0;
}

static inline int truth(PyObject* v, int* out)
{
    *out = PyObject_IsTrue(v);
    return *out < 0 ? -1 : 0;
}

static inline int arguments(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "%zd arguments are needed, not %zd", want, n);
    return -1;
}

static inline void keep(PyObject** at, PyObject* v)
{
    Py_INCREF(v);
    Py_XSETREF(*at, v);
}

/* The names of the tensors' methods, once. */
static inline int intern_names(void)
{
    struct { PyObject** at; const char* name; } names[] = {{&s_is_cuda, "is_cuda"}, {&s_is_contiguous, "is_contiguous"}, {&s_data_ptr, "data_ptr"},
                                                           {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_numel, "numel"},
                                                           {&s_element_size, "element_size"}};
    size_t i;
    for (i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!(*names[i].at = PyUnicode_InternFromString(names[i].name))) return -1;
    return 0;
}
