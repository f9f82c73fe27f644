/* Argument marshalling of the block operators for the Python binding.
 *
 * A call on one token runs for 3 to 6 us on the GPU and takes 3 us to launch; looking at six tensors from Python took 4 us more.
 * Here each is looked at once: its type, device, shape and strides, and its address, through the methods that tensors have
 * (nothing of torch is linked).  A tensor that is not what the call needs raises ValueError; nothing has been enqueued then.
 * The entry points' addresses are handed over once (init), as are torch's types and its current-stream function.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "slim.h"

static PyObject *s_dtype, *s_shape, *s_stride, *s_get_device, *s_data_ptr, *s_numel, *s_is_contiguous;
static PyObject *types[5];               /* fp16, bf16, fp32 (slim_dtype's numbers), uint8, E4M3 */
enum { U8 = 3, E4M3 = 4 };
static PyObject *stream_of;
static int (*call_norm)(const void *, int64_t, const void *, int64_t, const void *, int32_t, int32_t, int32_t, int32_t, float, void *,
                        int64_t, void *, int64_t, uint8_t *, float *, void *);
static int (*call_act)(const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, uint8_t *, float *, void *);
static int (*call_gemm)(const slim_block_fp8_layer *, const uint8_t *, const float *, int32_t, void *, int64_t, int32_t, void *, size_t,
                        void *);

static int refuse(const char *name, const char *why)
{
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s %s", name, why);
    return -1;
}

/* A method's result as a number; -2 with an exception set if it is none. */
static long long number(PyObject *t, PyObject *method)
{
    PyObject *r = PyObject_CallMethodNoArgs(t, method);
    if (!r) return -2;
    const long long v = PyLong_AsLongLong(r);
    Py_DECREF(r);
    return v == -1 && PyErr_Occurred() ? -2 : v;
}

static void *address(PyObject *t)
{
    PyObject *r = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!r) return NULL;
    void *p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return p;
}

/* The number of t's type in types[], -1 if it is none of them. */
static int type_of(PyObject *t, const char *name)
{
    PyObject *d = PyObject_GetAttr(t, s_dtype);
    if (!d) return -1;
    Py_DECREF(d);                        /* (torch's types live as long as torch) */
    for (int i = 0; i < 5; ++i)
        if (types[i] == d) return i;
    return refuse(name, "has a type that this call does not take");
}

static int pair(PyObject *tuple, long long *a, long long *b)
{
    if (!tuple) return -1;
    int ok = PyTuple_Check(tuple) && PyTuple_GET_SIZE(tuple) == 2;
    if (ok) {
        *a = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 0));
        *b = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, 1));
        ok = !PyErr_Occurred();
    }
    Py_DECREF(tuple);
    return ok ? 0 : -1;
}

typedef struct {
    void *p;
    int64_t ld;
    long long m, k;
    int type;
    long long device;
} matrix;

/* t as a matrix on a device whose rows have no gaps, whatever lies between them. */
static int rows(PyObject *t, const char *name, matrix *out)
{
    long long s0, s1;
    if ((out->type = type_of(t, name)) < 0) return -1;
    if ((out->device = number(t, s_get_device)) < 0) return refuse(name, "must be a device tensor");
    if (pair(PyObject_GetAttr(t, s_shape), &out->m, &out->k)) return refuse(name, "must be a matrix");
    if (pair(PyObject_CallMethodNoArgs(t, s_stride), &s0, &s1)) return refuse(name, "must be a matrix");
    if (s1 != 1 && out->k > 1) return refuse(name, "must have contiguous rows");
    if (out->m > INT32_MAX || out->k > INT32_MAX) return refuse(name, "is too large");
    out->ld = out->m > 1 || s0 > out->k ? s0 : out->k;          /* (the stride of a single row says nothing) */
    out->p = address(t);
    return PyErr_Occurred() ? -1 : 0;
}

/* The same of one that has to be like another. */
static int like(PyObject *t, const char *name, const matrix *other, matrix *out)
{
    if (rows(t, name, out)) return -1;
    if (out->type != other->type || out->device != other->device || out->m != other->m || out->k != other->k)
        return refuse(name, "must have the inputs' type, device and shape");
    return 0;
}

/* t's address; it has `count` elements of type a (or b) on the device, without gaps. */
static int whole(PyObject *t, const char *name, int a, int b, long long count, long long device, void **out)
{
    const int type = type_of(t, name);
    if (type < 0) return -1;
    if ((type != a && type != b) || number(t, s_numel) != count || number(t, s_get_device) != device)
        return refuse(name, "must have the type and size that the call needs, on the inputs' device");
    PyObject *c = PyObject_CallMethodNoArgs(t, s_is_contiguous);
    if (!c) return -1;
    Py_DECREF(c);
    if (c != Py_True) return refuse(name, "must be contiguous");
    *out = address(t);
    return PyErr_Occurred() ? -1 : 0;
}

static int stream(long long device, void **out)
{
    PyObject *d = PyLong_FromLongLong(device), *r = d ? PyObject_CallOneArg(stream_of, d) : NULL;
    Py_XDECREF(d);
    if (!r) return -1;
    *out = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return PyErr_Occurred() ? -1 : 0;
}

/* norm(X, gain, eps, residual, codes, scales, H, Y) -> status; gain, residual, H, Y may be None */
static PyObject *norm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 8) return PyErr_Format(PyExc_TypeError, "norm takes 8 arguments");
    matrix x, r = {0}, h = {0}, y = {0};
    void *gain = NULL, *codes, *scales, *st;
    int gain_type = SLIM_F32, status;
    if (rows(a[0], "X", &x)) return NULL;
    if (x.type != SLIM_F16 && x.type != SLIM_BF16) return refuse("X", "must be float16 or bfloat16"), NULL;
    const double eps = PyFloat_AsDouble(a[2]);
    if (eps == -1.0 && PyErr_Occurred()) return NULL;
    if (a[1] != Py_None) {
        if ((gain_type = type_of(a[1], "gain")) < 0 || whole(a[1], "gain", x.type, SLIM_F32, x.k, x.device, &gain)) return NULL;
    }
    if (a[3] != Py_None && like(a[3], "residual", &x, &r)) return NULL;
    if (a[6] != Py_None && like(a[6], "H", &x, &h)) return NULL;
    if (a[7] != Py_None && like(a[7], "Y", &x, &y)) return NULL;
    const long long kb = (x.k + 127) / 128;
    if (whole(a[4], "codes", U8, U8, x.m * kb * 128, x.device, &codes) || whole(a[5], "scales", SLIM_F32, SLIM_F32, x.m * kb, x.device, &scales) ||
        stream(x.device, &st))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    status = call_norm(x.p, x.ld, r.p, r.ld, gain, gain_type, x.type, (int32_t)x.m, (int32_t)x.k, (float)eps, h.p, h.ld, y.p, y.ld, codes, scales, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* act(G, U, act, codes, scales) -> status; U may be None */
static PyObject *act(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 5) return PyErr_Format(PyExc_TypeError, "act takes 5 arguments");
    matrix g, u = {0};
    void *codes, *scales, *st;
    int status;
    if (rows(a[0], "G", &g)) return NULL;
    if (g.type != SLIM_F16 && g.type != SLIM_BF16) return refuse("G", "must be float16 or bfloat16"), NULL;
    if (a[1] != Py_None && like(a[1], "U", &g, &u)) return NULL;
    const long kind = PyLong_AsLong(a[2]);
    if (kind == -1 && PyErr_Occurred()) return NULL;
    const long long kb = (g.k + 127) / 128;
    if (whole(a[3], "codes", U8, U8, g.m * kb * 128, g.device, &codes) || whole(a[4], "scales", SLIM_F32, SLIM_F32, g.m * kb, g.device, &scales) ||
        stream(g.device, &st))
        return NULL;
    Py_BEGIN_ALLOW_THREADS
    status = call_act(g.p, g.ld, u.p, u.ld, (int32_t)kind, g.type, (int32_t)g.m, (int32_t)g.k, codes, scales, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* gemm(layer's address, layer's device, the layer's codes and scales, codes, scales, Y, workspace) -> status, or 1 (nothing enqueued) where the layer's
   tensors are no longer where its struct says */
static PyObject *gemm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    (void)self;
    if (n != 8) return PyErr_Format(PyExc_TypeError, "gemm takes 8 arguments");
    const slim_block_fp8_layer *layer = PyLong_AsVoidPtr(a[0]);
    const long long device = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred() || !layer) return refuse("layer", "has no address"), NULL;
    matrix c, y;
    void *scales, *st;
    int status;
    const long long kb = ((long long)layer->k + 127) / 128, row_tiles = ((long long)layer->n + 63) / 64;
    const int stale = address(a[2]) != layer->codes || address(a[3]) != layer->scales || number(a[2], s_numel) != row_tiles * kb * 8192 ||
                      number(a[3], s_numel) != (row_tiles + 1) / 2 * kb;
    if (PyErr_Occurred()) return NULL;
    if (stale) return PyLong_FromLong(1);
    if (rows(a[4], "codes", &c)) return NULL;
    if ((c.type != U8 && c.type != E4M3) || c.device != device || c.k != kb * 128 || (c.m > 1 && c.ld != c.k))
        return refuse("codes", "must be contiguous uint8 [m][128 ceil(k / 128)] on the layer's device"), NULL;
    if (whole(a[5], "scales", SLIM_F32, SLIM_F32, c.m * kb, device, &scales)) return NULL;
    if (rows(a[6], "Y", &y)) return NULL;
    if (y.type > SLIM_F32 || y.device != device || y.m != c.m || y.k != layer->n)
        return refuse("Y", "must be a float16, bfloat16 or float32 matrix [m][n] on the layer's device"), NULL;
    const long long room = number(a[7], s_numel);
    void *ws;
    if (room < 0 || whole(a[7], "workspace", U8, U8, room, device, &ws) || stream(device, &st)) return NULL;
    Py_BEGIN_ALLOW_THREADS
    status = call_gemm(layer, c.p, scales, (int32_t)c.m, y.p, y.ld, y.type, ws, (size_t)room, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

/* init((fp16, bf16, fp32, uint8, e4m3), current-stream function, addresses of norm, act, gemm) */
static PyObject *init(PyObject *self, PyObject *args)
{
    (void)self;
    PyObject *t[5], *f, *p[3];
    if (!PyArg_ParseTuple(args, "(OOOOO)OOOO", &t[0], &t[1], &t[2], &t[3], &t[4], &f, &p[0], &p[1], &p[2])) return NULL;
    for (int i = 0; i < 5; ++i) {
        Py_INCREF(t[i]);
        Py_XSETREF(types[i], t[i]);
    }
    Py_INCREF(f);
    Py_XSETREF(stream_of, f);
    *(void **)&call_norm = PyLong_AsVoidPtr(p[0]);
    *(void **)&call_act = PyLong_AsVoidPtr(p[1]);
    *(void **)&call_gemm = PyLong_AsVoidPtr(p[2]);
    if (PyErr_Occurred()) return NULL;
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"init", init, METH_VARARGS, NULL},
                                {"norm", (PyCFunction)(void (*)(void))norm, METH_FASTCALL, NULL},
                                {"act", (PyCFunction)(void (*)(void))act, METH_FASTCALL, NULL},
                                {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_slim_args", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__slim_args(void)
{
    static const struct {
        PyObject **to;
        const char *name;
    } names[] = {{&s_dtype, "dtype"}, {&s_shape, "shape"}, {&s_stride, "stride"}, {&s_get_device, "get_device"}, {&s_data_ptr, "data_ptr"},
                 {&s_numel, "numel"}, {&s_is_contiguous, "is_contiguous"}};
    for (size_t i = 0; i < sizeof names / sizeof names[0]; ++i)
        if (!(*names[i].to = PyUnicode_InternFromString(names[i].name))) return NULL;
    return PyModule_Create(&module);
}
