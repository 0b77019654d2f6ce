// CPython binding of the gated recurrence over its C ABI (include/gated_recurrence.h), in the manner of attn_binding.cpp.
#include "torch_binding.h"

#include "gated_recurrence.h"

namespace {

void check(int status) { check(status, rec_last_error); }

int32_t type_code(at::ScalarType t)
{
    TORCH_CHECK_VALUE(t == at::kFloat || t == at::kBFloat16 || t == at::kHalf, "expected float32, bfloat16 or float16, got ", t);
    return t == at::kFloat ? REC_DT_F32 : t == at::kBFloat16 ? REC_DT_BF16 : REC_DT_F16;
}

// The address of [tokens, channels] whose channels are contiguous; *stride: elements between tokens.
void *rows(const char *name, const at::Tensor &t, int64_t tokens, int64_t channels, at::ScalarType type, int device, int64_t *stride)
{
    if (!is(t, {tokens, channels}, type, device))
        refuse(name, t, {tokens, channels}, type, device);
    TORCH_CHECK_VALUE(channels == 1 || t.stride(1) == 1, name, ": the channels of a token must be contiguous, got strides ", t.strides());
    *stride = tokens > 1 ? t.stride(0) : channels;
    return t.data_ptr();
}

// x, r, i, decay, which every operator begins with.
struct Inputs {
    rec_shape_t shape;
    int device;
    at::ScalarType type;
    int64_t T;
    const void *x, *r, *i;
    int64_t x_stride, r_stride, i_stride;
    const float *decay;
    at::TensorOptions options;
};
Inputs inputs(PyObject *const *args, PyObject *sharpness)
{
    const at::Tensor &x = tensor(args[0], "x"), &r = tensor(args[1], "r"), &i = tensor(args[2], "i"), &decay = tensor(args[3], "decay");
    Inputs in;
    in.device = on_current_device(x);
    in.type = x.scalar_type();
    in.options = x.options();
    TORCH_CHECK_VALUE(x.dim() == 2, "x: expected [tokens, channels], got ", x.sizes());
    in.T = x.size(0);
    const int64_t C = x.size(1);
    in.shape.channels = size32(C, "channels");
    in.shape.io_dtype = type_code(in.type);
    const double s = PyFloat_AsDouble(sharpness);
    if (s == -1.0 && PyErr_Occurred())
        throw python_error();
    in.shape.sharpness = (float)s;
    in.x = rows("x", x, in.T, C, in.type, in.device, &in.x_stride);
    in.r = rows("r", r, in.T, C, in.type, in.device, &in.r_stride);
    in.i = rows("i", i, in.T, C, in.type, in.device, &in.i_stride);
    in.decay = address<float>("decay", decay, {C}, at::kFloat, in.device);
    return in;
}
// Rows of states, or NULL for None.
float *states_or_null(PyObject *o, const char *name, int64_t n, const Inputs &in)
{
    return o == Py_None ? nullptr : address<float>(name, tensor(o, name), {n, in.shape.channels}, at::kFloat, in.device);
}
at::Tensor workspace_of(const Inputs &in, int64_t batch, int grads)
{
    size_t need = 0;
    check(rec_workspace_bytes(&in.shape, size32(batch, "batch"), in.T, grads, &need));
    return at::empty({(int64_t)need}, in.options.dtype(at::kByte));
}
typedef void Refusal(std::initializer_list<Named>);
void none_of(Refusal *refusal, PyObject *const *args, std::initializer_list<const char *> names)
{
    int k = 0;
    for (const char *name : names) {
        if (args[k] != Py_None)
            refusal({{name, &tensor(args[k], name)}});
        ++k;
    }
}

// (x, r, i, decay, cu_seqlens, sharpness, init_states | None, ckpt | None, out | None, save); what requires grad is the caller's business
PyObject *scan(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 10);
    none_of(no_tangents, args, {"x", "r", "i", "decay"});
    none_of(no_tangents, args + 6, {"init_states"});
    none_of(no_tangents, args + 8, {"out"});
    const Inputs in = inputs(args, args[5]);
    const at::Tensor &cu = tensor(args[4], "cu_seqlens");
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, in.device);
    const int64_t batch = cu.numel() - 1, C = in.shape.channels;
    TORCH_CHECK_VALUE(batch >= 0, "cu_seqlens: expected at least one value");
    const float *init = states_or_null(args[6], "init_states", batch, in);
    const int32_t *ckpt_at = nullptr;
    const at::TensorOptions floats = in.options.dtype(at::kFloat);
    at::Tensor ckpt_states, saved;
    int32_t n_ckpt = 0;
    if (args[7] != Py_None) {
        const at::Tensor &ckpt = tensor(args[7], "ckpt");
        ckpt_at = address<int32_t>("ckpt", ckpt, {-1}, at::kInt, in.device);
        n_ckpt = size32(ckpt.numel(), "ckpt");
        ckpt_states = at::empty({n_ckpt, C}, floats);
    }
    const int save = PyObject_IsTrue(args[9]);
    if (save < 0)
        throw python_error();
    const at::Tensor y = args[8] == Py_None ? at::empty({in.T, C}, in.options) : tensor(args[8], "out");
    int64_t y_stride;
    void *y_at = rows("out", y, in.T, C, in.type, in.device, &y_stride);
    const at::Tensor final_states = at::empty({batch, C}, floats);
    if (save)
        saved = at::empty({(in.T + REC_SAVED_EVERY - 1) / REC_SAVED_EVERY, C}, floats);
    const at::Tensor workspace = workspace_of(in, batch, 0);
    check(rec_scan(&in.shape, (int32_t)batch, in.T, in.x, in.x_stride, in.r, in.r_stride, in.i, in.i_stride, in.decay, cu_at, init, ckpt_at, n_ckpt, y_at, y_stride,
                   static_cast<float *>(final_states.data_ptr()), n_ckpt ? static_cast<float *>(ckpt_states.data_ptr()) : nullptr,
                   save ? static_cast<float *>(saved.data_ptr()) : nullptr, workspace.data_ptr(), workspace.numel(), stream(in.device)));
    if (args[8] != Py_None)
        written(y);
    return tuple_of({&y, &final_states, &ckpt_states, &saved});
    END_HANDLE_TH_ERRORS
}

// (x, r, i, decay, cu_seqlens, sharpness, init_states | None, saved | None, dy | None, d_final | None, wants d_init)
PyObject *scan_grads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 11);
    none_of(no_tangents, args, {"x", "r", "i", "decay"});
    none_of(no_tangents, args + 6, {"init_states", "saved", "dy", "d_final"});
    const Inputs in = inputs(args, args[5]);
    const at::Tensor &cu = tensor(args[4], "cu_seqlens");
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, in.device);
    const int64_t batch = cu.numel() - 1, C = in.shape.channels;
    TORCH_CHECK_VALUE(batch >= 0, "cu_seqlens: expected at least one value");
    const float *init = states_or_null(args[6], "init_states", batch, in);
    const float *saved = states_or_null(args[7], "saved", (in.T + REC_SAVED_EVERY - 1) / REC_SAVED_EVERY, in);
    int64_t dy_stride = C;
    const void *dy = args[8] == Py_None ? nullptr : rows("dy", tensor(args[8], "dy"), in.T, C, in.type, in.device, &dy_stride);
    const float *d_final = states_or_null(args[9], "d_final", batch, in);
    const int wants_init = PyObject_IsTrue(args[10]);
    if (wants_init < 0)
        throw python_error();
    const at::TensorOptions floats = in.options.dtype(at::kFloat);
    const at::Tensor dx = at::empty({in.T, C}, in.options), dr = at::empty({in.T, C}, in.options), di = at::empty({in.T, C}, in.options), d_decay = at::empty({C}, floats);
    at::Tensor d_init;
    if (wants_init)
        d_init = at::empty({batch, C}, floats);
    const at::Tensor workspace = workspace_of(in, batch, saved ? 1 : 2);
    check(rec_scan_grads(&in.shape, (int32_t)batch, in.T, in.x, in.x_stride, in.r, in.r_stride, in.i, in.i_stride, in.decay, cu_at, init, saved, dy, dy_stride, d_final,
                         dx.data_ptr(), dr.data_ptr(), di.data_ptr(), static_cast<float *>(d_decay.data_ptr()),
                         wants_init ? static_cast<float *>(d_init.data_ptr()) : nullptr, workspace.data_ptr(), workspace.numel(), stream(in.device)));
    return tuple_of({&dx, &dr, &di, &d_decay, &d_init});
    END_HANDLE_TH_ERRORS
}

// (x, r, i, decay, states, sharpness, out | None)
PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 7);
    none_of(no_gradients, args, {"x", "r", "i", "decay", "states"});
    none_of(no_gradients, args + 6, {"out"});
    const Inputs in = inputs(args, args[5]);
    const at::Tensor &states = tensor(args[4], "states");
    float *states_at = address<float>("states", states, {in.T, in.shape.channels}, at::kFloat, in.device);
    const at::Tensor y = args[6] == Py_None ? at::empty({in.T, in.shape.channels}, in.options) : tensor(args[6], "out");
    int64_t y_stride;
    void *y_at = rows("out", y, in.T, in.shape.channels, in.type, in.device, &y_stride);
    check(rec_step(&in.shape, size32(in.T, "batch"), in.x, in.x_stride, in.r, in.r_stride, in.i, in.i_stride, in.decay, states_at, y_at, y_stride, stream(in.device)));
    written(states);
    if (args[6] != Py_None)
        written(y);
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// (x, r, i, decay, states, cu_seqlens, parents, sharpness, out | None)
PyObject *step_tree(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 9);
    none_of(no_gradients, args, {"x", "r", "i", "decay", "states"});
    none_of(no_gradients, args + 8, {"out"});
    const Inputs in = inputs(args, args[7]);
    const at::Tensor &cu = tensor(args[5], "cu_seqlens");
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, in.device);
    const int64_t batch = cu.numel() - 1, C = in.shape.channels;
    TORCH_CHECK_VALUE(batch >= 0, "cu_seqlens: expected at least one value");
    const float *states = address<float>("states", tensor(args[4], "states"), {batch, C}, at::kFloat, in.device);
    const int32_t *parents = address<int32_t>("parents", tensor(args[6], "parents"), {in.T}, at::kInt, in.device);
    const at::Tensor y = args[8] == Py_None ? at::empty({in.T, C}, in.options) : tensor(args[8], "out"), nodes = at::empty({in.T, C}, in.options.dtype(at::kFloat));
    int64_t y_stride;
    void *y_at = rows("out", y, in.T, C, in.type, in.device, &y_stride);
    check(rec_step_tree(&in.shape, size32(batch, "batch"), in.T, in.x, in.x_stride, in.r, in.r_stride, in.i, in.i_stride, in.decay, states, cu_at, parents, y_at, y_stride,
                        static_cast<float *>(nodes.data_ptr()), stream(in.device)));
    if (args[8] != Py_None)
        written(y);
    return tuple_of({&y, &nodes});
    END_HANDLE_TH_ERRORS
}

// (states, node_states, cu_seqlens, path, counts)
PyObject *keep_states(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 5);
    none_of(no_gradients, args, {"states", "node_states"});
    const at::Tensor &states = tensor(args[0], "states"), &nodes = tensor(args[1], "node_states"), &cu = tensor(args[2], "cu_seqlens"), &path = tensor(args[3], "path");
    const int device = on_current_device(states);
    TORCH_CHECK_VALUE(states.dim() == 2, "states: expected [batch, channels], got ", states.sizes());
    const int64_t batch = states.size(0), C = states.size(1), T = path.numel();
    float *states_at = address<float>("states", states, {batch, C}, at::kFloat, device);
    const float *nodes_at = address<float>("node_states", nodes, {T, C}, at::kFloat, device);
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {batch + 1}, at::kInt, device), *path_at = address<int32_t>("path", path, {-1}, at::kInt, device);
    const int32_t *counts_at = address<int32_t>("counts", tensor(args[4], "counts"), {batch}, at::kInt, device);
    check(rec_keep_states(size32(C, "channels"), size32(batch, "batch"), T, states_at, nodes_at, cu_at, path_at, counts_at, stream(device)));
    written(states);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"scan", (PyCFunction)(void (*)(void))scan, METH_FASTCALL, nullptr},
    {"scan_grads", (PyCFunction)(void (*)(void))scan_grads, METH_FASTCALL, nullptr},
    {"step", (PyCFunction)(void (*)(void))step, METH_FASTCALL, nullptr},
    {"step_tree", (PyCFunction)(void (*)(void))step_tree, METH_FASTCALL, nullptr},
    {"keep_states", (PyCFunction)(void (*)(void))keep_states, METH_FASTCALL, nullptr},
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rec_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rec_binding() { return PyModule_Create(&module); }
