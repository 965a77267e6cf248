// The operators of pwlq_block.h for Python, on tensors: _pwlq_block.pack_rows and the others that block.py documents.
//
// A call of a few rows is bound by the host: checking ten tensors' types, shapes and strides and allocating three outputs from
// Python took 12 of an adapter call's 17 us.  Here they are C++ members of the tensor.  Each function checks what it is
// given (ValueError), allocates what is not given, and makes one call of the library; a status other than PWLQ_OK is raised as
// pwlq.PwlqError.  `stream` is the handle of a stream.  The interpreter's lock is released during the library's call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <utility>

#include "../../../include/pwlq.h"
#include "../../../include/pwlq_block.h"

namespace {

using at::ScalarType;
using at::Tensor;

PyObject *g_error = nullptr;           // pwlq.PwlqError

template <typename... A> [[noreturn]] void refuse(const char *format, A... a)
{
    PyErr_Format(PyExc_ValueError, format, a...);
    throw python_error();
}

// A tensor, or NULL for None.
const Tensor *tensor(const char *name, PyObject *o)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        throw python_error();
    }
    return &THPVariable_Unpack(o);
}
const Tensor &needed(const char *name, PyObject *o)
{
    const Tensor *t = tensor(name, o);
    if (!t) refuse("%s is None", name);
    return *t;
}

// What autograd would have to follow through a forward call is refused: the result would be a constant to it.
void untracked(const char *backward, std::initializer_list<std::pair<const char *, const Tensor *>> tensors)
{
    if (!at::GradMode::is_enabled()) return;
    for (const auto &[name, t] : tensors)
        if (t && t->requires_grad())
            refuse("%s requires gradients, and this call records nothing for autograd: %s is its backward pass; call it under torch.no_grad()", name,
                   backward);
}

int type_of(ScalarType t)
{
    return t == at::kFloat ? PWLQ_F32 : t == at::kBFloat16 ? PWLQ_BF16 : t == at::kHalf ? PWLQ_F16 : t == at::kChar ? PWLQ_I8 : -1;
}
bool is_float(ScalarType t) { return t == at::kFloat || t == at::kBFloat16 || t == at::kHalf; }
ScalarType dtype_of(PyObject *o, ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "dtype must be a torch.dtype");
        throw python_error();
    }
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

// What every tensor of a call is checked against.  The device is the current one: the work is launched there, on its stream.
struct Call {
    at::Device device;
    int64_t T;

    Call(const char *name, const Tensor &x) : device(x.device()), T(0)
    {
        if (!x.is_cuda() || x.dim() != 2) refuse("%s must be a matrix on the GPU", name);
        const at::Device current = c10::impl::VirtualGuardImpl(at::kCUDA).getDevice();
        if (device != current) refuse("%s is on GPU %d, and the current device is GPU %d", name, (int)device.index(), (int)current.index());
        T = x.size(0);
    }
    Tensor make(at::IntArrayRef sizes, ScalarType type) const { return at::empty(sizes, at::TensorOptions().dtype(type).device(device)); }

    void dense(const char *name, const Tensor *t, at::IntArrayRef sizes, ScalarType type) const
    {
        if (t && !(t->device() == device && t->scalar_type() == type && t->sizes() == sizes && t->is_contiguous()))
            refuse("%s must be contiguous, of the sizes, the type and the device that go with the other arguments", name);
    }
    const float *floats(const char *name, const Tensor *t, at::IntArrayRef sizes) const
    {
        dense(name, t, sizes, at::kFloat);
        return t ? static_cast<const float *>(t->data_ptr()) : nullptr;
    }
    // `type` and `other`: the types taken; `factors`: steps may go with a float type.
    pwlq_rows rows(const char *name, const Tensor *t, int64_t cols, ScalarType type, ScalarType other, const Tensor *step = nullptr,
                   bool factors = false) const
    {
        pwlq_rows r = {nullptr, nullptr, 0, 0};
        if (!t) {
            if (step) refuse("%s is None and has steps", name);
            return r;
        }
        const ScalarType is = t->scalar_type();
        if (!(t->device() == device && (is == type || is == other) && t->dim() == 2 && t->size(0) == T && t->size(1) == cols))
            refuse("%s must be a matrix of the sizes, the type and the device that go with the other arguments", name);
        if ((cols > 1 && t->stride(1) != 1) || (T > 1 && t->stride(0) < cols))
            refuse("%s must have its columns next to each other, and rows that do not overlap", name);
        if (is == at::kChar ? !step : (step && !factors)) refuse("%s needs its steps where it is int8, and has none else", name);
        r.data = t->data_ptr();
        r.step = const_cast<float *>(floats("the steps", step, {T}));
        r.stride = T > 1 ? t->stride(0) : cols;
        r.type = type_of(is);
        return r;
    }
    // A workspace of the caller's, or one for this call; none where none is needed.
    void *room(PyObject *given, size_t need, Tensor &keep, size_t &bytes) const
    {
        if (const Tensor *t = tensor("workspace", given)) {
            if (t->device() != device || !t->is_contiguous()) refuse("workspace must be contiguous and on the device of the other arguments");
            bytes = t->nbytes();
            return t->data_ptr();
        }
        bytes = need;
        if (!need) return nullptr;
        keep = make({(int64_t)need}, at::kByte);
        return keep.data_ptr();
    }
};

void *stream_of(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw python_error();
    return p;
}
float real(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}
void count(const char *name, Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return;
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, %zd given", name, want, got);
    throw python_error();
}
template <typename F> void call(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    if (rc == PWLQ_OK) return;
    PyObject *e = g_error ? PyObject_CallFunction(g_error, "is", rc, pwlq_last_error()) : nullptr;
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw python_error();
}

PyObject *wrap(Tensor t) { return t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None); }
template <typename... A> PyObject *tuple(A... a)
{
    PyObject *all = PyTuple_New(sizeof...(a));
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(all, i++, wrap(std::move(a))), ...);
    return all;
}

// x, codes or None, step or None, stream
PyObject *pack_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("pack_rows", n, 4);
    const Tensor &x = needed("x", a[0]);
    const Call c("x", x);
    const int64_t K = x.size(1);
    if (!is_float(x.scalar_type())) refuse("x must be float32, bfloat16 or float16");
    const pwlq_rows rows = c.rows("x", &x, K, x.scalar_type(), x.scalar_type());
    const Tensor *out = tensor("codes", a[1]), *out_step = tensor("step", a[2]);
    Tensor codes = out ? *out : c.make({c.T, K}, at::kChar), step = out_step ? *out_step : c.make({c.T}, at::kFloat);
    c.dense("codes", &codes, {c.T, K}, at::kChar);
    c.dense("step", &step, {c.T}, at::kFloat);
    void *stream = stream_of(a[3]);
    call([&] { return pwlq_pack_rows(&rows, c.T, K, (int8_t *)codes.data_ptr(), (float *)step.data_ptr(), stream); });
    return tuple(codes, step);
    END_HANDLE_TH_ERRORS
}

// codes, step, dtype, out or None, stream
PyObject *unpack_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("unpack_rows", n, 5);
    const Tensor &codes = needed("codes", a[0]), &step = needed("step", a[1]);
    const Call c("codes", codes);
    const int64_t K = codes.size(1);
    c.dense("codes", &codes, {c.T, K}, at::kChar);
    c.dense("step", &step, {c.T}, at::kFloat);
    const Tensor *given = tensor("out", a[3]);
    Tensor out = given ? *given : c.make({c.T, K}, dtype_of(a[2], at::kFloat));
    if (!is_float(out.scalar_type())) refuse("out must be float32, bfloat16 or float16");
    const pwlq_rows rows = c.rows("out", &out, K, out.scalar_type(), out.scalar_type());
    void *stream = stream_of(a[4]);
    call([&] { return pwlq_unpack_rows((const int8_t *)codes.data_ptr(), (const float *)step.data_ptr(), c.T, K, &rows, stream); });
    return wrap(out);
    END_HANDLE_TH_ERRORS
}

// The gate's pointer; its rows.
const void *gate_of(const Call &c, const Tensor *gate, int64_t D, ScalarType type, int64_t &gate_rows)
{
    gate_rows = 0;
    if (!gate) return nullptr;
    if (gate->dim() != 2) refuse("gate must be a matrix");
    gate_rows = gate->size(0);
    c.dense("gate", gate, {gate_rows, D}, type);
    return gate->data_ptr();
}

// x, f or None, pre_weight, post_weight or None, gate or None, alpha, eps, pack, stream
PyObject *norm_block(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("norm_block", n, 9);
    const Tensor &x = needed("x", a[0]), *f = tensor("f", a[1]), &pre = needed("pre_weight", a[2]);
    const Tensor *post = tensor("post_weight", a[3]), *gate = tensor("gate", a[4]);
    const Call c("x", x);
    untracked("norm_block_backward", {{"x", &x}, {"f", f}, {"pre_weight", &pre}, {"post_weight", post}, {"gate", gate}});
    const ScalarType stream_type = x.scalar_type(), type = f ? f->scalar_type() : stream_type;
    if (!is_float(stream_type) || !is_float(type)) refuse("x and f must be float32, bfloat16 or float16");
    const int pack = PyObject_IsTrue(a[7]);
    if (pack < 0) throw python_error();
    pwlq_norm_args args = {};
    args.T = c.T;
    args.D = x.size(1);
    args.x = c.rows("x", &x, args.D, stream_type, stream_type);
    args.f = c.rows("f", f, args.D, type, type);
    args.pre_weight = c.floats("pre_weight", &pre, {args.D});
    args.post_weight = c.floats("post_weight", post, {args.D});
    args.gate = gate_of(c, gate, args.D, type, args.gate_rows);
    args.alpha = real(a[5]);
    args.eps = real(a[6]);
    void *stream = stream_of(a[8]);
    Tensor x_out = f ? c.make({c.T, args.D}, stream_type) : x, u = c.make({c.T, args.D}, pack ? at::kChar : type), step;
    if (pack) step = c.make({c.T}, at::kFloat);
    if (f) args.x_out = c.rows("x_out", &x_out, args.D, stream_type, stream_type);
    args.u = c.rows("u", &u, args.D, u.scalar_type(), u.scalar_type(), pack ? &step : nullptr);
    call([&] { return pwlq_norm_block(&args, stream); });
    return pack ? tuple(x_out, u, step) : tuple(x_out, u);
    END_HANDLE_TH_ERRORS
}

// du or None, dx_out or None, x_out, f or None, pre_weight, post_weight or None, gate or None, alpha, eps, x_step or None,
// f_step or None, dtype or None, workspace or None, stream
PyObject *norm_block_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("norm_block_backward", n, 14);
    const Tensor *du = tensor("du", a[0]), *dx_out = tensor("dx_out", a[1]), &x_out = needed("x_out", a[2]), *f = tensor("f", a[3]);
    const Tensor &pre = needed("pre_weight", a[4]), *post = tensor("post_weight", a[5]), *gate = tensor("gate", a[6]);
    if (!du && !dx_out) refuse("du and dx_out are both None");
    const Call c("x_out", x_out);
    const bool kept = x_out.scalar_type() == at::kChar;
    const ScalarType stream_type = dx_out ? dx_out->scalar_type() : kept ? du->scalar_type() : x_out.scalar_type();
    // 8-bit checkpoints do not say the type that f had: the gate has it too, or the caller says it
    const ScalarType said = dtype_of(a[11], stream_type);
    const ScalarType type = du ? du->scalar_type() : !f ? stream_type : !kept ? f->scalar_type() : gate ? gate->scalar_type() : said;
    if (!is_float(stream_type) || !is_float(type)) refuse("gradients of rows must be float32, bfloat16 or float16");
    pwlq_norm_backward_args args = {};
    args.T = c.T;
    args.D = x_out.size(1);
    args.du = c.rows("du", du, args.D, type, type);
    args.dx_out = c.rows("dx_out", dx_out, args.D, stream_type, stream_type);
    const ScalarType x_type = kept ? at::kChar : stream_type, f_type = kept ? at::kChar : type;
    args.x_out = c.rows("x_out", &x_out, args.D, x_type, x_type, tensor("x_step", a[9]));
    args.f = c.rows("f", f, args.D, f_type, f_type, tensor("f_step", a[10]));
    args.pre_weight = c.floats("pre_weight", &pre, {args.D});
    args.post_weight = c.floats("post_weight", post, {args.D});
    args.gate = gate_of(c, gate, args.D, type, args.gate_rows);
    args.alpha = real(a[7]);
    args.eps = real(a[8]);
    void *stream = stream_of(a[13]);
    Tensor dx = c.make({c.T, args.D}, stream_type), df, d_pre = c.make({args.D}, at::kFloat), d_post, d_gate, keep;
    args.dx = c.rows("dx", &dx, args.D, stream_type, stream_type);
    args.d_pre = (float *)d_pre.data_ptr();
    if (f) {
        df = c.make({c.T, args.D}, type);
        args.df = c.rows("df", &df, args.D, type, type);
    }
    if (post) {
        d_post = c.make({args.D}, at::kFloat);
        args.d_post = (float *)d_post.data_ptr();
    }
    if (gate) {
        d_gate = c.make({args.gate_rows, args.D}, at::kFloat);
        args.d_gate = (float *)d_gate.data_ptr();
    }
    size_t bytes = 0;
    void *room = c.room(a[12], pwlq_norm_block_backward_workspace_bytes(c.T, args.D, args.gate_rows), keep, bytes);
    call([&] { return pwlq_norm_block_backward(&args, room, bytes, stream); });
    return tuple(dx, df, d_pre, d_post, d_gate);
    END_HANDLE_TH_ERRORS
}

// What the adapters' calls have in common, into args: T, K, N, R, adapters, the weights, ids and scale.
template <typename Args>
ScalarType adapters(const Call &c, Args &args, int64_t K, const Tensor &down, const Tensor &up, const Tensor &ids, const Tensor &scale)
{
    const ScalarType type = down.scalar_type();
    if (down.dim() != 3 || up.dim() != 3 || !is_float(type)) refuse("down [adapters, R, K] and up [adapters, R, N] must be float32, bfloat16 or float16");
    const int64_t n = up.size(0), R = up.size(1);
    args.T = c.T;
    args.K = K;
    args.N = up.size(2);
    if (n > INT32_MAX || R > INT32_MAX) refuse("up has too many adapters or ranks");
    args.adapters = (int)n;
    args.R = (int)R;
    args.weight_type = type_of(type);
    c.dense("down", &down, {n, R, K}, type);
    c.dense("up", &up, {n, R, args.N}, type);
    c.dense("ids", &ids, {c.T}, at::kInt);
    args.down = down.data_ptr();
    args.up = up.data_ptr();
    args.ids = (const int32_t *)ids.data_ptr();
    args.scale = c.floats("scale", &scale, {n});
    return type;
}

// x, down, up, ids, scale, base or None, x_step or None, base_step or None, dtype or None, out or None, workspace or None, stream
PyObject *adapter(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("adapter", n, 12);
    const Tensor &x = needed("x", a[0]);
    const Call c("x", x);
    const int64_t K = x.size(1);
    const Tensor &down = needed("down", a[1]), &up = needed("up", a[2]), &scale = needed("scale", a[4]);
    const Tensor *base = tensor("base", a[5]), *x_step = tensor("x_step", a[6]), *base_step = tensor("base_step", a[7]);
    const Tensor *given = tensor("out", a[9]);
    untracked("adapter_backward", {{"x", &x}, {"down", &down}, {"up", &up}, {"scale", &scale}, {"base", base}, {"x_step", x_step},
                                   {"base_step", base_step}, {"out", given}});
    pwlq_adapter_args args = {};
    const ScalarType type = adapters(c, args, K, down, up, needed("ids", a[3]), scale);
    args.x = c.rows("x", &x, K, type, at::kChar, x_step);
    args.base = c.rows("base", base, args.N, type, at::kFloat, base_step, true);
    void *stream = stream_of(a[11]);
    Tensor out = given ? *given : c.make({c.T, args.N}, dtype_of(a[8], type)), h = c.make({c.T, args.R}, at::kFloat), keep;
    args.out = c.rows("out", &out, args.N, type, at::kFloat);
    args.h = (float *)h.data_ptr();
    size_t bytes = 0;
    void *room = c.room(a[10], pwlq_adapter_workspace_bytes(c.T, K, args.R), keep, bytes);
    call([&] { return pwlq_adapter(&args, room, bytes, stream); });
    return tuple(out, h);
    END_HANDLE_TH_ERRORS
}

// dy, x, down, up, ids, scale, h, x_step or None, dx_base or None, dtype or None, workspace or None, stream
PyObject *adapter_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("adapter_backward", n, 12);
    const Tensor &x = needed("x", a[1]);
    const Call c("x", x);
    const int64_t K = x.size(1);
    pwlq_adapter_backward_args args = {};
    const ScalarType type = adapters(c, args, K, needed("down", a[2]), needed("up", a[3]), needed("ids", a[4]), needed("scale", a[5]));
    args.dy = c.rows("dy", &needed("dy", a[0]), args.N, type, type);
    args.x = c.rows("x", &x, K, type, at::kChar, tensor("x_step", a[7]));
    const Tensor *base = tensor("dx_base", a[8]);
    args.dx_base = c.rows("dx_base", base, K, type, at::kFloat);
    args.h = c.floats("h", &needed("h", a[6]), {c.T, args.R});
    void *stream = stream_of(a[11]);
    Tensor dx = c.make({c.T, K}, base ? base->scalar_type() : dtype_of(a[9], type)), keep;
    Tensor d_down = c.make({args.adapters, args.R, K}, at::kFloat), d_up = c.make({args.adapters, args.R, args.N}, at::kFloat);
    args.dx = c.rows("dx", &dx, K, type, at::kFloat);
    args.d_down = (float *)d_down.data_ptr();
    args.d_up = (float *)d_up.data_ptr();
    size_t bytes = 0;
    void *room = c.room(a[10], pwlq_adapter_backward_workspace_bytes(c.T, K, args.N, args.R, args.adapters), keep, bytes);
    call([&] { return pwlq_adapter_backward(&args, room, bytes, stream); });
    return tuple(d_down, d_up, dx);
    END_HANDLE_TH_ERRORS
}

// The exception of a refused call.
PyObject *raises(PyObject *, PyObject *error)
{
    Py_XSETREF(g_error, Py_NewRef(error));
    return Py_NewRef(Py_None);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {METHOD(pack_rows), METHOD(unpack_rows), METHOD(norm_block), METHOD(norm_block_backward), METHOD(adapter),
                           METHOD(adapter_backward), {"raises", raises, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_pwlq_block", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__pwlq_block(void) { return PyModule_Create(&g_module); }
