/* Argument marshalling of the operators at the decoder's two ends and of the update of its matrices, as a Python extension module: as sdl_operators.c does it
 * for those between.  Each function takes the arguments of the binding's function of the same name, in that order, and returns the library's status.
 *
 * Nothing is kept from one call for the next. */
#include "sdl_arguments.h"

#define ENTRIES(X) X(sdl_embedding) X(sdl_embedding_backward) X(sdl_cross_entropy) X(sdl_cross_entropy_backward) X(sdl_orthogonalize)

/* the library's functions, by address (the library is loaded by the binding) */
#define DECLARE(name) static __typeof__(&name) p_##name;
ENTRIES(DECLARE)

#define MOST_STEPS 64

/* [batch, tokens, width] from the right, without heads */
static int rows(PyObject* t, Operand* o)
{
    if (operand(t, o) < 0) return -1;
    if (o->dims > 3) {
        PyErr_SetString(PyExc_ValueError, "a tensor of one to three dimensions is needed");
        return -1;
    }
    return 0;
}

/* One token for every row of x. */
static int tokens_of(PyObject* t, const Operand* x, const char* what, void** at, sdl_index_t* index)
{
    PyObject* dtype;
    if (t == Py_None) {
        PyErr_Format(PyExc_ValueError, "%s: a tensor is needed", what);
        return -1;
    }
    if (on_device(t) < 0 || !(dtype = type_of(t))) return -1;
    if (dtype != t_int32 && dtype != t_int64) {
        PyErr_Format(PyExc_ValueError, "%s: int32 or int64 is needed", what);
        return -1;
    }
    *index = dtype == t_int64 ? SDL_INDEX_INT64 : SDL_INDEX_INT32;
    return flat(t, (unsigned long long)x->shape[0] * x->shape[1], dtype, what, at);
}

/* [vocab, width], rows at any distance */
static int table_of(PyObject* t, Operand* o, sdl_dtype_t* dtype)
{
    if (operand(t, o) < 0 || dtype_number(o->dtype, dtype) < 0) return -1;
    if (o->dims != 2) {
        PyErr_SetString(PyExc_ValueError, "a table of two dimensions is needed");
        return -1;
    }
    return 0;
}

static int same_width(const Operand* a, const Operand* b)
{
    if (a->shape[3] == b->shape[3]) return 0;
    PyErr_SetString(PyExc_ValueError, "rows of another width than the table's");
    return -1;
}

/* table, tokens, out, scale, stream */
static PyObject* py_sdl_embedding(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Operand table, out;
    void *tokens, *stream;
    sdl_dtype_t table_dtype, dtype;
    sdl_index_t index;
    float scale;
    (void)self;
    if (arguments(n, 5) < 0 || table_of(a[0], &table, &table_dtype) < 0 || rows(a[2], &out) < 0 || dtype_number(out.dtype, &dtype) < 0 || same_width(&table, &out) < 0 ||
        tokens_of(a[1], &out, "tokens", &tokens, &index) < 0 || real(a[3], &scale) < 0 || stream_of(a[4], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_embedding(table.view.data, table.view.stride_token, table.shape[1], table.shape[3], table_dtype, tokens, index, out.shape[0],
                                           out.shape[1], scale, &out.view, dtype, stream));
}

/* d_out, tokens, d_table, workspace, scale, stream */
static PyObject* py_sdl_embedding_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Operand table, d_out;
    void *tokens, *work, *stream;
    sdl_dtype_t table_dtype, dtype;
    sdl_index_t index;
    size_t bytes;
    float scale;
    (void)self;
    if (arguments(n, 6) < 0 || rows(a[0], &d_out) < 0 || dtype_number(d_out.dtype, &dtype) < 0 || table_of(a[2], &table, &table_dtype) < 0 ||
        same_width(&table, &d_out) < 0 || tokens_of(a[1], &d_out, "tokens", &tokens, &index) < 0 || space(a[3], &work, &bytes) < 0 || real(a[4], &scale) < 0 ||
        stream_of(a[5], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_embedding_backward(&d_out.view, dtype, tokens, index, d_out.shape[0], d_out.shape[1], scale, table.view.data,
                                                    table.view.stride_token, table.shape[1], table.shape[3], table_dtype, work, bytes, stream));
}

typedef struct {
    Operand x, d;
    sdl_dtype_t dtype;
    sdl_index_t index;
    void* targets;
    unsigned long long n;
    float smoothing, z;
    int gradient;
} Loss;

static int loss_of(PyObject* logits, PyObject* targets, PyObject* d_logits, PyObject* smoothing, PyObject* z, Loss* l)
{
    if (rows(logits, &l->x) < 0 || dtype_number(l->x.dtype, &l->dtype) < 0 || tokens_of(targets, &l->x, "targets", &l->targets, &l->index) < 0 ||
        real(smoothing, &l->smoothing) < 0 || real(z, &l->z) < 0)
        return -1;
    l->gradient = d_logits != Py_None;
    l->n = (unsigned long long)l->x.shape[0] * l->x.shape[1];
    return l->gradient ? operand_like(d_logits, &l->x, &l->d) : 0;
}

/* logits, targets, loss, lse, d_logits, d_loss, smoothing, z, stream */
static PyObject* py_sdl_cross_entropy(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Loss l;
    void *loss, *lse, *d_loss, *stream;
    (void)self;
    if (arguments(n, 9) < 0 || loss_of(a[0], a[1], a[4], a[6], a[7], &l) < 0 || flat(a[2], l.n, t_float32, "loss", &loss) < 0 ||
        flat(a[3], l.n, t_float32, "lse", &lse) < 0 || flat(a[5], l.n, t_float32, "d_loss", &d_loss) < 0 || stream_of(a[8], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_cross_entropy(&l.x.view, l.x.shape[0], l.x.shape[1], l.x.shape[3], l.dtype, l.targets, l.index, l.smoothing, l.z, loss, lse,
                                               d_loss, l.gradient ? &l.d.view : NULL, stream));
}

/* logits, targets, lse, d_logits, d_loss, smoothing, z, stream */
static PyObject* py_sdl_cross_entropy_backward(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Loss l;
    void *lse, *d_loss, *stream;
    (void)self;
    if (arguments(n, 8) < 0 || loss_of(a[0], a[1], a[3], a[5], a[6], &l) < 0 || flat(a[2], l.n, t_float32, "lse", &lse) < 0 ||
        flat(a[4], l.n, t_float32, "d_loss", &d_loss) < 0 || stream_of(a[7], &stream) < 0)
        return NULL;
    return PyLong_FromLong(p_sdl_cross_entropy_backward(&l.x.view, l.x.shape[0], l.x.shape[1], l.x.shape[3], l.dtype, l.targets, l.index, l.smoothing, l.z, lse,
                                                        d_loss, l.gradient ? &l.d.view : NULL, stream));
}

/* A list or tuple of (a, b, c). */
static int coefficients_of(PyObject* v, float* out, uint32_t* steps)
{
    PyObject *all = PySequence_Fast(v, "coefficients are a list of (a, b, c)"), *each, *item;
    Py_ssize_t i, k, n;
    if (!all) return -1;
    n = PySequence_Fast_GET_SIZE(all);
    if (n > MOST_STEPS) {
        PyErr_Format(PyExc_ValueError, "at most %d steps", MOST_STEPS);
        goto bad;
    }
    for (i = 0; i < n; ++i) {
        /* a number's own code may change the list that it stands in */
        if (i >= PySequence_Fast_GET_SIZE(all)) {
            PyErr_SetString(PyExc_ValueError, "the coefficients changed while they were read");
            goto bad;
        }
        item = PySequence_Fast_GET_ITEM(all, i);
        Py_INCREF(item);
        each = PySequence_Tuple(item);
        Py_DECREF(item);
        if (!each) goto bad;
        if (PyTuple_GET_SIZE(each) != 3) {
            PyErr_SetString(PyExc_ValueError, "three coefficients a step are needed");
            Py_DECREF(each);
            goto bad;
        }
        for (k = 0; k < 3; ++k)
            if (real(PyTuple_GET_ITEM(each, k), &out[3 * i + k]) < 0) {
                Py_DECREF(each);
                goto bad;
            }
        Py_DECREF(each);
    }
    Py_DECREF(all);
    *steps = (uint32_t)n;
    return 0;
bad:
    Py_DECREF(all);
    return -1;
}

/* x, out, workspace, coefficients, eps, scale, stream */
static PyObject* py_sdl_orthogonalize(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    Operand x, out;
    void *work, *stream;
    sdl_dtype_t dtype, out_dtype;
    size_t bytes;
    float coefficients[3 * MOST_STEPS], eps, scale;
    uint32_t steps;
    int i;
    (void)self;
    if (arguments(n, 7) < 0 || rows(a[0], &x) < 0 || dtype_number(x.dtype, &dtype) < 0 || rows(a[1], &out) < 0 || dtype_number(out.dtype, &out_dtype) < 0 ||
        space(a[2], &work, &bytes) < 0 || coefficients_of(a[3], coefficients, &steps) < 0 || real(a[4], &eps) < 0 || real(a[5], &scale) < 0 ||
        stream_of(a[6], &stream) < 0)
        return NULL;
    for (i = 0; i < 4; ++i)
        if (x.dims < 2 || x.dims != out.dims || x.shape[i] != out.shape[i]) {
            PyErr_SetString(PyExc_ValueError, "x and out are [rows, cols] or [batch, rows, cols], both of them");
            return NULL;
        }
    return PyLong_FromLong(p_sdl_orthogonalize(&x.view, x.shape[0], x.shape[1], x.shape[3], dtype, coefficients, steps, eps, scale, &out.view, out_dtype, work, bytes,
                                               stream));
}

/* setup({name: address}, (float32, bfloat16, int32, int64), stream, is_initialized, get_device, raw_stream) */
static PyObject* setup(PyObject* self, PyObject* args)
{
    PyObject *table, *f32, *bf16, *i32, *i64, *stream, *initialized, *device, *raw, *v;
    (void)self;
    if (!PyArg_ParseTuple(args, "O!(OOOO)OOOO", &PyDict_Type, &table, &f32, &bf16, &i32, &i64, &stream, &initialized, &device, &raw)) return NULL;
#define TAKE(name)                                                                                  \
    v = PyDict_GetItemString(table, #name);                                                         \
    if (!v) return PyErr_Format(PyExc_KeyError, #name);                                             \
    p_##name = (__typeof__(p_##name))(uintptr_t)PyLong_AsUnsignedLongLong(v);                       \
    if (PyErr_Occurred()) return NULL;
    ENTRIES(TAKE)
    keep(&t_float32, f32);
    keep(&t_bfloat16, bf16);
    keep(&t_int32, i32);
    keep(&t_int64, i64);
    keep(&f_stream, stream);
    keep(&f_initialized, initialized);
    keep(&f_device, device);
    keep(&f_raw_stream, raw);
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, NULL},
static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, NULL}, ENTRIES(METHOD){NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_training", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__training(void)
{
    if (intern_names() < 0) return NULL;
    return PyModule_Create(&module);
}
