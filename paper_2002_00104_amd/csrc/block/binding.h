// What the bindings of the operators share: tensors' types, shapes and strides checked, outputs and workspaces allocated, a
// call of the library made, and its status raised as pwlq.PwlqError.
#pragma once

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
// `backward`: the call that is its backward pass, or NULL if it has none.
void untracked(const char *backward, std::initializer_list<std::pair<const char *, const Tensor *>> tensors)
{
    if (!at::GradMode::is_enabled()) return;
    for (const auto &[name, t] : tensors)
        if (t && t->requires_grad()) {
            if (!backward)
                refuse("%s requires gradients, and this call records nothing for autograd and has no backward pass; call it under torch.no_grad()", name);
            refuse("%s requires gradients, and this call records nothing for autograd: %s is its backward pass; call it under torch.no_grad()", name,
                   backward);
        }
}

int type_of(ScalarType t)
{
    return t == at::kFloat ? PWLQ_F32 : t == at::kBFloat16 ? PWLQ_BF16 : t == at::kHalf ? PWLQ_F16 : t == at::kChar ? PWLQ_I8 : -1;
}
[[maybe_unused]] bool is_float(ScalarType t) { return t == at::kFloat || t == at::kBFloat16 || t == at::kHalf; }
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

    Call(const char *name, const Tensor &x, int dims = 2) : device(x.device()), T(0)
    {
        if (!x.is_cuda() || x.dim() != dims) refuse(dims == 2 ? "%s must be a matrix on the GPU" : "%s must be on the GPU, with %d dimensions", name, dims);
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

// The exception of a refused call.
PyObject *raises(PyObject *, PyObject *error)
{
    Py_XSETREF(g_error, Py_NewRef(error));
    return Py_NewRef(Py_None);
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}

} // namespace
