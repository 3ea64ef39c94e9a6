/* Argument marshalling of the inner step's operators, as a Python extension module: strided tensors into views, their shapes and types
 * checked, and that they are on a device (on which one is the caller's to see to, as everywhere in the binding).  Each function takes the arguments of the binding's function of the same name, in that order, and returns the
 * library's status.  A norm of one token takes 10.3 us with this in Python and ctypes, of which the launch is 4.5.
 *
 * Nothing is kept from one call for the next. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <stdint.h>

#include "sdl.h"

#define ENTRIES(X) X(sdl_layer_norm) X(sdl_layer_norm_backward) X(sdl_rotary) X(sdl_attention) X(sdl_attention_backward)

/* the library's functions, by address (the library is loaded by the binding) */
#define DECLARE(name) static __typeof__(&name) p_##name;
ENTRIES(DECLARE)

static PyObject *s_is_cuda, *s_is_contiguous, *s_data_ptr, *s_shape, *s_stride, *s_dtype, *s_numel, *s_element_size;
static PyObject *t_float32, *t_bfloat16, *t_int32, *t_float64;        /* torch's types */
static PyObject *f_stream, *f_initialized, *f_device, *f_raw_stream;

typedef struct {
    sdl_view_t view;
    uint32_t shape[4];      /* batch, tokens, heads, width */
    Py_ssize_t dims;
    PyObject* dtype;        /* borrowed: one of the four above, or None for another */
} Operand;

static int number(PyObject* v, long long* out)
{
    *out = PyLong_AsLongLong(v);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
}

/* a method without arguments that gives a number */
static int ask(PyObject* t, PyObject* name, long long* out)
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

static int on_device(PyObject* t)
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

static PyObject* type_of(PyObject* t)
{
    PyObject *r = PyObject_GetAttr(t, s_dtype), *known;
    if (!r) return NULL;
    known = r == t_float32 || r == t_bfloat16 || r == t_int32 || r == t_float64 ? r : Py_None;
    Py_DECREF(r);           /* the module keeps the four */
    return known;
}

static int dtype_number(PyObject* dtype, sdl_dtype_t* out)
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
static int operand(PyObject* t, Operand* o)
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
static int operand_like(PyObject* t, const Operand* like, Operand* o)
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
static int flat(PyObject* t, unsigned long long numel, PyObject* dtype, const char* what, void** out)
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

static int space(PyObject* t, void** at, size_t* bytes)
{
    long long n, each;
    *bytes = 0;
    if (flat(t, 0, NULL, "workspace", at) < 0) return -1;
    if (t == Py_None) return 0;
    if (ask(t, s_numel, &n) < 0 || ask(t, s_element_size, &each) < 0) return -1;
    *bytes = (size_t)n * (size_t)each;
    return 0;
}

static int stream_of(PyObject* v, void** out)
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

static int real(PyObject* v, float* out)
{
    const double x = PyFloat_AsDouble(v);
    if (x == -1.0 && PyErr_Occurred()) return -1;
    *out = (float)x;
    return 0;
}

static int integer(PyObject* v, int32_t* out)
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

static int truth(PyObject* v, int* out)
{
    *out = PyObject_IsTrue(v);
    return *out < 0 ? -1 : 0;
}

static int arguments(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want) return 0;
    PyErr_Format(PyExc_TypeError, "%zd arguments are needed, not %zd", want, n);
    return -1;
}

static unsigned long long rows_of(const Operand* x) { return (unsigned long long)x->shape[0] * x->shape[1] * x->shape[2]; }

/* The parameter arrays of a norm have one type, the first one's that is there. */
static int params(PyObject* const* ts, const int* at, int n, uint32_t width, void** out, sdl_dtype_t* number_of)
{
    PyObject* dtype = NULL;
    int i;
    *number_of = SDL_DTYPE_FP32;
    for (i = 0; i < n && !dtype; ++i)
        if (ts[at[i]] != Py_None) {
            if (on_device(ts[at[i]]) < 0) return -1;
            dtype = type_of(ts[at[i]]);
            if (!dtype || dtype_number(dtype, number_of) < 0) return -1;
        }
    for (i = 0; i < n; ++i)
        if (flat(ts[at[i]], width, dtype, "parameters of a norm", &out[i]) < 0) return -1;
    return 0;
}

/* x, weight, bias, eps, y, mean, rstd, stream */
static PyObject* py_sdl_layer_norm(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    static const int which[2] = {1, 2};
    Operand x, y;
    void *p[2], *mean, *rstd, *stream;
    sdl_dtype_t dtype, param_dtype;
    float eps;
    (void)self;
    if (arguments(n, 8) < 0 || operand(a[0], &x) < 0 || dtype_number(x.dtype, &dtype) < 0 || params(a, which, 2, x.shape[3], p, &param_dtype) < 0 ||
        real(a[3], &eps) < 0 || operand_like(a[4], &x, &y) < 0 || flat(a[5], rows_of(&x), t_float32, "mean", &mean) < 0 ||
        flat(a[6], rows_of(&x), t_float32, "rstd", &rstd) < 0 || stream_of(a[7], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_layer_norm(&x.view, x.shape[0], x.shape[1], x.shape[2], x.shape[3], dtype, p[0], p[1], param_dtype, eps, &y.view,
                                            mean, rstd, stream));
}

/* dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, stream */
static PyObject* py_sdl_layer_norm_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    static const int which[3] = {2, 6, 7};
    Operand x, dy, dx;
    void *p[3], *mean, *rstd, *work, *stream;
    sdl_dtype_t dtype, param_dtype;
    size_t bytes;
    (void)self;
    if (arguments(n, 10) < 0 || operand(a[1], &x) < 0 || dtype_number(x.dtype, &dtype) < 0 || operand_like(a[0], &x, &dy) < 0 ||
        params(a, which, 3, x.shape[3], p, &param_dtype) < 0 || flat(a[3], rows_of(&x), t_float32, "mean", &mean) < 0 ||
        flat(a[4], rows_of(&x), t_float32, "rstd", &rstd) < 0 || operand_like(a[5], &x, &dx) < 0 || space(a[8], &work, &bytes) < 0 ||
        stream_of(a[9], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_layer_norm_backward(&dy.view, &x.view, x.shape[0], x.shape[1], x.shape[2], x.shape[3], dtype, p[0], param_dtype, mean, rstd,
                                                     &dx.view, p[1], p[2], work, bytes, stream));
}

/* x, positions, frequencies, out, layout, scale, inverse, first_position, stream */
static PyObject* py_sdl_rotary(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Operand x, out;
    void *positions, *f, *stream;
    sdl_dtype_t dtype;
    long long half;
    int32_t layout, first;
    int inverse;
    float scale;
    (void)self;
    if (arguments(n, 9) < 0 || operand(a[0], &x) < 0 || dtype_number(x.dtype, &dtype) < 0 || operand_like(a[3], &x, &out) < 0 ||
        flat(a[1], (unsigned long long)x.shape[0] * x.shape[1], t_int32, "positions", &positions) < 0 || ask(a[2], s_numel, &half) < 0 ||
        flat(a[2], (unsigned long long)half, t_float64, "frequencies", &f) < 0 || integer(a[4], &layout) < 0 || real(a[5], &scale) < 0 ||
        truth(a[6], &inverse) < 0 || integer(a[7], &first) < 0 || stream_of(a[8], &stream) < 0)
        return NULL;
    if (half > INT32_MAX / 2) half = INT32_MAX / 2;          /* more than any width: the library refuses it */
    return PyLong_FromLong(p_sdl_rotary(&x.view, x.shape[0], x.shape[1], x.shape[2], x.shape[3], dtype, (uint32_t)(2 * half), (sdl_rotary_layout_t)layout,
                                        positions, first, f, scale, inverse, &out.view, stream));
}

typedef struct {
    Operand q, k, v;
    sdl_dtype_t dtype;
    float scale;
    int causal;
    void *q_len, *k_len;
    unsigned long long stats;
} Problem;

static int problem(PyObject* q, PyObject* k, PyObject* v, PyObject* scale, PyObject* causal, PyObject* q_len, PyObject* k_len, Problem* p)
{
    if (operand(q, &p->q) < 0 || dtype_number(p->q.dtype, &p->dtype) < 0 || operand(k, &p->k) < 0) return -1;
    if (p->q.dims != 4 || p->k.dims != 4 || p->q.shape[0] != p->k.shape[0] || p->q.shape[3] != p->k.shape[3]) {
        PyErr_SetString(PyExc_ValueError, "attention takes q [batch, queries, heads, width] and k, v [batch, keys, kv_heads, width]");
        return -1;
    }
    if (p->k.dtype != p->q.dtype) {
        PyErr_Format(PyExc_ValueError, "a tensor of another type where %R is needed", p->q.dtype);
        return -1;
    }
    if (operand_like(v, &p->k, &p->v) < 0 || truth(causal, &p->causal) < 0 || real(scale, &p->scale) < 0) return -1;
    p->stats = (unsigned long long)p->q.shape[0] * p->q.shape[1] * p->q.shape[2];
    return flat(q_len, p->q.shape[0], t_int32, "q_len", &p->q_len) < 0 || flat(k_len, p->q.shape[0], t_int32, "k_len", &p->k_len) < 0 ? -1 : 0;
}

#define SHAPE(p) p.q.shape[0], p.q.shape[1], p.k.shape[1], p.q.shape[2], p.k.shape[2], p.q.shape[3]

/* q, k, v, out, lse, workspace, scale, causal, q_len, k_len, stream */
static PyObject* py_sdl_attention(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Problem p;
    Operand out;
    void *lse, *work, *stream;
    size_t bytes;
    (void)self;
    if (arguments(n, 11) < 0 || problem(a[0], a[1], a[2], a[6], a[7], a[8], a[9], &p) < 0 || operand_like(a[3], &p.q, &out) < 0 ||
        flat(a[4], p.stats, t_float32, "lse", &lse) < 0 || space(a[5], &work, &bytes) < 0 || stream_of(a[10], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_attention(&p.q.view, &p.k.view, &p.v.view, SHAPE(p), p.dtype, p.scale, p.causal, p.q_len, p.k_len, &out.view, lse, work,
                                           bytes, stream));
}

/* d_out, q, k, v, out, lse, dq, dk, dv, workspace, scale, causal, q_len, k_len, stream */
static PyObject* py_sdl_attention_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Problem p;
    Operand out, d_out, dq, dk, dv;
    void *lse, *work, *stream;
    size_t bytes;
    (void)self;
    if (arguments(n, 15) < 0 || problem(a[1], a[2], a[3], a[10], a[11], a[12], a[13], &p) < 0 || operand_like(a[0], &p.q, &d_out) < 0 ||
        operand_like(a[4], &p.q, &out) < 0 || flat(a[5], p.stats, t_float32, "lse", &lse) < 0 || operand_like(a[6], &p.q, &dq) < 0 ||
        operand_like(a[7], &p.k, &dk) < 0 || operand_like(a[8], &p.k, &dv) < 0 || space(a[9], &work, &bytes) < 0 || stream_of(a[14], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_attention_backward(&d_out.view, &p.q.view, &p.k.view, &p.v.view, &out.view, lse, SHAPE(p), p.dtype, p.scale, p.causal,
                                                    p.q_len, p.k_len, &dq.view, &dk.view, &dv.view, work, bytes, stream));
}

static void keep(PyObject** at, PyObject* v)
{
    Py_INCREF(v);
    Py_XSETREF(*at, v);
}

/* setup({name: address}, (float32, bfloat16, int32, float64), stream, is_initialized, get_device, raw_stream) */
static PyObject* setup(PyObject* self, PyObject* args)
{
    PyObject *table, *f32, *bf16, *i32, *f64, *stream, *initialized, *device, *raw, *v;
    (void)self;
    if (!PyArg_ParseTuple(args, "O!(OOOO)OOOO", &PyDict_Type, &table, &f32, &bf16, &i32, &f64, &stream, &initialized, &device, &raw)) return NULL;
#define TAKE(name)                                                                                  \
    v = PyDict_GetItemString(table, #name);                                                         \
    if (!v) return PyErr_Format(PyExc_KeyError, #name);                                             \
    p_##name = (__typeof__(p_##name))(uintptr_t)PyLong_AsUnsignedLongLong(v);                       \
    if (PyErr_Occurred()) return NULL;
    ENTRIES(TAKE)
    keep(&t_float32, f32);
    keep(&t_bfloat16, bf16);
    keep(&t_int32, i32);
    keep(&t_float64, f64);
    keep(&f_stream, stream);
    keep(&f_initialized, initialized);
    keep(&f_device, device);
    keep(&f_raw_stream, raw);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL},
static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, NULL}, ENTRIES(METHOD){NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_operators", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__operators(void)
{
    struct { PyObject** at; const char* name; } names[] = {{&s_is_cuda, "is_cuda"}, {&s_is_contiguous, "is_contiguous"}, {&s_data_ptr, "data_ptr"},
                                                           {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_dtype, "dtype"}, {&s_numel, "numel"},
                                                           {&s_element_size, "element_size"}};
    size_t i;
    for (i = 0; i < sizeof(names) / sizeof(names[0]); ++i)
        if (!(*names[i].at = PyUnicode_InternFromString(names[i].name))) return NULL;
    return PyModule_Create(&module);
}
