/* Argument marshalling of the inner step's operators, as a Python extension module: strided tensors into views, their shapes and types
 * checked, and that they are on a device (on which one is the caller's to see to, as everywhere in the binding).  Each function takes the arguments of the binding's function of the same name, in that order, and returns the
 * library's status.  A norm of one token takes 10.3 us with this in Python and ctypes, of which the launch is 4.5.
 *
 * Nothing is kept from one call for the next. */
#include "sdl_arguments.h"

#define ENTRIES(X) X(sdl_layer_norm) X(sdl_layer_norm_backward) X(sdl_rotary) X(sdl_attention) X(sdl_attention_backward)

/* the library's functions, by address (the library is loaded by the binding) */
#define DECLARE(name) static __typeof__(&name) p_##name;
ENTRIES(DECLARE)

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
    if (intern_names() < 0) return NULL;
    return PyModule_Create(&module);
}
