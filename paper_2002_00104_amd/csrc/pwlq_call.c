/* Calls of the library from Python without ctypes: _pwlq_call.search, .quantize and .linear_i8, and the operators of
 * pwlq_block.h, whose argument structures are filled here: .pack_rows, .unpack_rows, .norm_block, .norm_block_backward,
 * .adapter and .adapter_backward.
 *
 * A call of one small tensor is bound by the host: of 5.0 us for an inner product of 8 x 256 x 64, the launch
 * included, 0.9 us were ctypes converting sixteen arguments and 1.4 us the binding around it.
 * A function takes the address of the library's function (ctypes knows it), then that function's arguments;
 * where it has a pointer, a tensor (its data_ptr() is asked for here), or None where the library takes NULL.
 * An integer is taken for the function and for the stream only: in the place of a tensor it would reach a
 * kernel as a device address.  The interpreter's lock is released during the call.  Returns the library's status. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include "../../include/pwlq_block.h"

static PyObject *data_ptr_name;

static int64_t whole(PyObject *o, int *bad)
{
    const long long v = *bad ? 0 : PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) *bad = 1;
    return v;
}

static int small(PyObject *o, int *bad)
{
    const int64_t v = whole(o, bad);
    if (!*bad && v != (int)v) {
        PyErr_SetString(PyExc_OverflowError, "an argument does not fit an int");
        *bad = 1;
    }
    return (int)v;
}

static float real(PyObject *o, int *bad)
{
    const double v = *bad ? 0.0 : PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) *bad = 1;
    return (float)v;
}

/* The function or the stream. */
static void *handle(PyObject *o, int *bad)
{
    void *p;
    if (*bad) return NULL;
    if (!PyLong_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "the function and the stream are integers");
        *bad = 1;
        return NULL;
    }
    p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) *bad = 1;
    return p;
}

static void *function(PyObject *o, int *bad)
{
    void *p = handle(o, bad);
    if (!p && !*bad) {
        PyErr_SetString(PyExc_TypeError, "the function is NULL");
        *bad = 1;
    }
    return p;
}

static void *tensor(PyObject *o, int *bad)
{
    PyObject *v = *bad ? NULL : PyObject_CallMethodNoArgs(o, data_ptr_name);
    void *p = NULL;
    if (v) {
        p = PyLong_AsVoidPtr(v);
        Py_DECREF(v);
    }
    if (!p && PyErr_Occurred()) *bad = 1;
    return p;
}

static int count(const char *name, Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return 1;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, %zd given", name, want, got);
    return 0;
}

#define FN(i) function(a[i], &bad)
#define TENSOR(i) tensor(a[i], &bad)
#define TENSOR_OR_NONE(i) (a[i] == Py_None ? NULL : tensor(a[i], &bad))
#define STREAM(i) handle(a[i], &bad)
#define INT(i) small(a[i], &bad)
#define I64(i) whole(a[i], &bad)
#define F32(i) real(a[i], &bad)

typedef int (*SearchFn)(const void *, int64_t, int64_t, int, int, int, void *, void *, void *, void *, void *, size_t,
                        void *);

/* fn, w, C, K, bits, n_cand, mode, p_star, m, k_star, mse, workspace, workspace_bytes, stream */
static PyObject *call_search(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    (void)self;
    if (!count("search", n, 14)) return NULL;
    SearchFn fn = (SearchFn)FN(0);
    void *w = TENSOR(1), *p = TENSOR(7), *m = TENSOR(8), *k = TENSOR(9), *mse = TENSOR(10), *ws = TENSOR(11), *stream = STREAM(13);
    const int64_t C = I64(2), K = I64(3), bytes = I64(12);
    const int bits = INT(4), cand = INT(5), mode = INT(6);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(w, C, K, bits, cand, mode, p, m, k, mse, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*QuantizeFn)(const void *, int64_t, int64_t, int, int, const void *, const void *, void *, void *, void *,
                          void *);

/* fn, w, C, K, bits, mode, p_star, m, codes, flags, w_hat, stream */
static PyObject *call_quantize(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    (void)self;
    if (!count("quantize", n, 12)) return NULL;
    QuantizeFn fn = (QuantizeFn)FN(0);
    void *w = TENSOR(1), *p = TENSOR(6), *m = TENSOR(7), *codes = TENSOR(8), *flags = TENSOR(9), *hat = TENSOR_OR_NONE(10),
         *stream = STREAM(11);
    const int64_t C = I64(2), K = I64(3);
    const int bits = INT(4), mode = INT(5);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(w, C, K, bits, mode, p, m, codes, flags, hat, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*LinearFn)(const void *, int64_t, int64_t, float, float, const void *, const void *, int64_t, int,
                        const void *, const void *, void *, void *, void *, size_t, void *);

/* fn, xq, M, K, s_x, z_x, packed_codes, packed_flags, N, bits, p, m, y, acc, workspace, workspace_bytes, stream */
static PyObject *call_linear(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    (void)self;
    if (!count("linear_i8", n, 17)) return NULL;
    LinearFn fn = (LinearFn)FN(0);
    void *xq = TENSOR(1), *codes = TENSOR(6), *flags = TENSOR(7), *p = TENSOR(10), *m = TENSOR(11), *y = TENSOR(12), *acc = TENSOR_OR_NONE(13),
         *ws = TENSOR(14), *stream = STREAM(16);
    const int64_t M = I64(2), K = I64(3), N = I64(8), bytes = I64(15);
    const float s_x = F32(4), z_x = F32(5);
    const int bits = INT(9);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(xq, M, K, s_x, z_x, codes, flags, N, bits, p, m, y, acc, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

/* Rows take four arguments: the tensor, or None where they are left out, its type, its stride and its steps, or None. */
static pwlq_rows rows(PyObject *const *a, int *bad)
{
    pwlq_rows r = {NULL, NULL, 0, 0};
    if (a[0] != Py_None) {
        r.data = tensor(a[0], bad);
        r.type = small(a[1], bad);
        r.stride = whole(a[2], bad);
        r.step = a[3] == Py_None ? NULL : tensor(a[3], bad);
    }
    return r;
}
#define ROWS(i) rows(a + (i), &bad)

typedef int (*PackFn)(const pwlq_rows *, int64_t, int64_t, void *, void *, void *);

/* fn, x[4], T, K, codes, step, stream */
static PyObject *call_pack_rows(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    (void)self;
    if (!count("pack_rows", n, 10)) return NULL;
    PackFn fn = (PackFn)FN(0);
    const pwlq_rows x = ROWS(1);
    const int64_t T = I64(5), K = I64(6);
    void *codes = TENSOR_OR_NONE(7), *step = TENSOR_OR_NONE(8), *stream = STREAM(9);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&x, T, K, codes, step, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*UnpackFn)(const void *, const void *, int64_t, int64_t, const pwlq_rows *, void *);

/* fn, codes, step, T, K, out[4], stream */
static PyObject *call_unpack_rows(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    (void)self;
    if (!count("unpack_rows", n, 10)) return NULL;
    UnpackFn fn = (UnpackFn)FN(0);
    void *codes = TENSOR_OR_NONE(1), *step = TENSOR_OR_NONE(2), *stream = STREAM(9);
    const int64_t T = I64(3), K = I64(4);
    const pwlq_rows out = ROWS(5);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(codes, step, T, K, &out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*NormFn)(const pwlq_norm_args *, void *);

/* fn, T, D, x[4], f[4], x_out[4], u[4], post_weight, pre_weight, gate, gate_rows, alpha, eps, stream */
static PyObject *call_norm_block(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    pwlq_norm_args args;
    (void)self;
    if (!count("norm_block", n, 26)) return NULL;
    NormFn fn = (NormFn)FN(0);
    args.T = I64(1);
    args.D = I64(2);
    args.x = ROWS(3);
    args.f = ROWS(7);
    args.x_out = ROWS(11);
    args.u = ROWS(15);
    args.post_weight = TENSOR_OR_NONE(19);
    args.pre_weight = TENSOR_OR_NONE(20);
    args.gate = TENSOR_OR_NONE(21);
    args.gate_rows = I64(22);
    args.alpha = F32(23);
    args.eps = F32(24);
    void *stream = STREAM(25);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&args, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*NormBackwardFn)(const pwlq_norm_backward_args *, void *, size_t, void *);

/* fn, T, D, du[4], dx_out[4], x_out[4], f[4], dx[4], df[4], post_weight, pre_weight, gate, gate_rows, alpha, eps, d_pre,
 * d_post, d_gate, workspace, workspace_bytes, stream */
static PyObject *call_norm_block_backward(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    pwlq_norm_backward_args args;
    (void)self;
    if (!count("norm_block_backward", n, 39)) return NULL;
    NormBackwardFn fn = (NormBackwardFn)FN(0);
    args.T = I64(1);
    args.D = I64(2);
    args.du = ROWS(3);
    args.dx_out = ROWS(7);
    args.x_out = ROWS(11);
    args.f = ROWS(15);
    args.dx = ROWS(19);
    args.df = ROWS(23);
    args.post_weight = TENSOR_OR_NONE(27);
    args.pre_weight = TENSOR_OR_NONE(28);
    args.gate = TENSOR_OR_NONE(29);
    args.gate_rows = I64(30);
    args.alpha = F32(31);
    args.eps = F32(32);
    args.d_pre = TENSOR_OR_NONE(33);
    args.d_post = TENSOR_OR_NONE(34);
    args.d_gate = TENSOR_OR_NONE(35);
    void *ws = TENSOR_OR_NONE(36), *stream = STREAM(38);
    const int64_t bytes = I64(37);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&args, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*AdapterFn)(const pwlq_adapter_args *, void *, size_t, void *);

/* fn, T, K, N, R, adapters, weight_type, down, up, ids, scale, x[4], base[4], out[4], h, workspace, workspace_bytes, stream */
static PyObject *call_adapter(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    pwlq_adapter_args args;
    (void)self;
    if (!count("adapter", n, 27)) return NULL;
    AdapterFn fn = (AdapterFn)FN(0);
    args.T = I64(1);
    args.K = I64(2);
    args.N = I64(3);
    args.R = INT(4);
    args.adapters = INT(5);
    args.weight_type = INT(6);
    args.down = TENSOR_OR_NONE(7);
    args.up = TENSOR_OR_NONE(8);
    args.ids = TENSOR_OR_NONE(9);
    args.scale = TENSOR_OR_NONE(10);
    args.x = ROWS(11);
    args.base = ROWS(15);
    args.out = ROWS(19);
    args.h = TENSOR_OR_NONE(23);
    void *ws = TENSOR_OR_NONE(24), *stream = STREAM(26);
    const int64_t bytes = I64(25);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&args, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

typedef int (*AdapterBackwardFn)(const pwlq_adapter_backward_args *, void *, size_t, void *);

/* fn, T, K, N, R, adapters, weight_type, down, up, ids, scale, dy[4], x[4], dx_base[4], dx[4], h, d_down, d_up, workspace,
 * workspace_bytes, stream */
static PyObject *call_adapter_backward(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int bad = 0, rc;
    pwlq_adapter_backward_args args;
    (void)self;
    if (!count("adapter_backward", n, 33)) return NULL;
    AdapterBackwardFn fn = (AdapterBackwardFn)FN(0);
    args.T = I64(1);
    args.K = I64(2);
    args.N = I64(3);
    args.R = INT(4);
    args.adapters = INT(5);
    args.weight_type = INT(6);
    args.down = TENSOR_OR_NONE(7);
    args.up = TENSOR_OR_NONE(8);
    args.ids = TENSOR_OR_NONE(9);
    args.scale = TENSOR_OR_NONE(10);
    args.dy = ROWS(11);
    args.x = ROWS(15);
    args.dx_base = ROWS(19);
    args.dx = ROWS(23);
    args.h = TENSOR_OR_NONE(27);
    args.d_down = TENSOR_OR_NONE(28);
    args.d_up = TENSOR_OR_NONE(29);
    void *ws = TENSOR_OR_NONE(30), *stream = STREAM(32);
    const int64_t bytes = I64(31);
    if (bad) return NULL;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(&args, ws, (size_t)bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))call_##name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {
    {"search", (PyCFunction)(void (*)(void))call_search, METH_FASTCALL, NULL},
    {"quantize", (PyCFunction)(void (*)(void))call_quantize, METH_FASTCALL, NULL},
    {"linear_i8", (PyCFunction)(void (*)(void))call_linear, METH_FASTCALL, NULL},
    METHOD(pack_rows),
    METHOD(unpack_rows),
    METHOD(norm_block),
    METHOD(norm_block_backward),
    METHOD(adapter),
    METHOD(adapter_backward),
    {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pwlq_call", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__pwlq_call(void)
{
    data_ptr_name = PyUnicode_InternFromString("data_ptr");
    return data_ptr_name ? PyModule_Create(&module) : NULL;
}
