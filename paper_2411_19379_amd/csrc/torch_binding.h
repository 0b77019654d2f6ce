// What the CPython bindings of the operators share: checks of tensors and numbers, errors, the current stream.
#pragma once

#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <sstream>

namespace {

PyObject *g_error_class = nullptr;  // the module's error (code, message)

// Raises what a negative status stands for.
void check(int status, const char *(*last_error)(void))
{
    if (status == 0)
        return;
    PyObject *e = PyObject_CallFunction(g_error_class ? g_error_class : PyExc_RuntimeError, "is", status, last_error());
    if (e) {
        PyErr_SetObject((PyObject *)Py_TYPE(e), e);
        Py_DECREF(e);
    }
    throw python_error();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, ": expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

[[noreturn]] void refuse(const char *name, const at::Tensor &t, std::initializer_list<int64_t> sizes, at::ScalarType type, int device)
{
    std::ostringstream want;
    const char *sep = "(";
    for (int64_t n : sizes) {
        want << sep;
        n < 0 ? want << "any" : want << n;
        sep = ", ";
    }
    TORCH_CHECK_VALUE(false, name, ": expected a contiguous ", type, " tensor of shape ", want.str(), ") on cuda:", device, ", got ",
                      t.scalar_type(), " ", t.sizes(), " with strides ", t.strides(), " on ", t.device());
}

bool is(const at::Tensor &t, std::initializer_list<int64_t> sizes, at::ScalarType type, int device)
{
    if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != device || t.dim() != (int64_t)sizes.size())
        return false;
    int64_t i = 0;
    for (int64_t n : sizes) {
        if (n >= 0 && t.size(i) != n)
            return false;
        ++i;
    }
    return true;
}

// The address of a contiguous tensor of these sizes (negative: any).
template <typename T = void> T *address(const char *name, const at::Tensor &t, std::initializer_list<int64_t> sizes, at::ScalarType type, int device)
{
    if (!is(t, sizes, type, device) || !t.is_contiguous())
        refuse(name, t, sizes, type, device);
    return static_cast<T *>(t.data_ptr());
}

struct Named {
    const char *name;
    const at::Tensor *t;
};
// Nothing hands on the tangents of forward-mode differentiation, which torch.no_grad() does not stop: a result without one would drop
// it in silence.
void no_tangents(std::initializer_list<Named> all)
{
    if (!c10::AutogradState::get_tls_state().get_fw_grad_mode())
        return;
    for (const Named &n : all)
        TORCH_CHECK_VALUE(!n.t->_fw_grad(0).defined(), n.name, " has a tangent, and this operator has no forward-mode derivative: detach it");
}
// There is no backward pass: where a graph is recorded, a result outside it would drop gradients in silence.
void no_gradients(std::initializer_list<Named> all)
{
    no_tangents(all);
    if (!c10::GradMode::is_enabled())
        return;
    for (const Named &n : all)
        TORCH_CHECK_VALUE(!n.t->requires_grad(), n.name, " requires grad, and this operator has no backward pass: call it under torch.no_grad(), or detach");
}

// A tensor of the caller's has been written: what autograd keeps of it is out of date.  (Inference tensors have no version.)
void written(const at::Tensor &t)
{
    if (!t.is_inference())
        t.unsafeGetTensorImpl()->bump_version();
}

int on_current_device(const at::Tensor &t)
{
    TORCH_CHECK_VALUE(t.is_cuda() && t.get_device() == c10::hip::current_device(), "expected tensors on the current CUDA device, got ", t.device());
    return (int)t.get_device();
}

inline int32_t int32_of(PyObject *o, const char *name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred())
        throw python_error();
    TORCH_CHECK_VALUE(v >= -0x7fffffffLL - 1 && v <= 0x7fffffffLL, name, " does not fit 32 bits");
    return (int32_t)v;
}

int32_t size32(int64_t n, const char *name)
{
    TORCH_CHECK_VALUE(n >= 0 && n <= 0x7fffffff, name, " does not fit 32 bits");
    return (int32_t)n;
}

void arguments(Py_ssize_t got, Py_ssize_t want)
{
    TORCH_CHECK_TYPE(got == want, "expected ", want, " arguments, got ", got);
}

void *stream(int device) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream(); }

PyObject *tuple_of(std::initializer_list<const at::Tensor *> all)
{
    PyObject *r = PyTuple_New((Py_ssize_t)all.size());
    if (!r)
        throw python_error();
    Py_ssize_t i = 0;
    for (const at::Tensor *t : all) {
        if (!t->defined())
            Py_INCREF(Py_None);
        PyTuple_SET_ITEM(r, i++, t->defined() ? THPVariable_Wrap(*t) : Py_None);
    }
    return r;
}

PyObject *set_error_class(PyObject *, PyObject *c)
{
    Py_INCREF(c);
    Py_XDECREF(g_error_class);
    g_error_class = c;
    Py_RETURN_NONE;
}

}  // namespace
