// CPython binding of the attention operators over their C ABI (include/attn_cache.h): checks of tensors, outputs and workspace
// from torch's allocator, the current stream.  A decode step of a layer is a few microseconds of GPU work, and the same steps
// written in Python with ctypes took longer than that (append 10.7 us and attention 10.0 us per call in front of the launches).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <sstream>

#include "attn_cache.h"

namespace {

PyObject *g_error_class = nullptr;  // AttnError(code, message)

// Raises what a negative status stands for.
void check(int status)
{
    if (status == ATTN_OK)
        return;
    PyObject *e = PyObject_CallFunction(g_error_class ? g_error_class : PyExc_RuntimeError, "is", status, attn_last_error());
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

// The address of [tokens, heads, dim] whose heads are contiguous; *stride: elements between tokens.
void *rows(const char *name, const at::Tensor &t, std::initializer_list<int64_t> sizes, at::ScalarType type, int device, int64_t *stride)
{
    if (!is(t, sizes, type, device))
        refuse(name, t, sizes, type, device);
    const int64_t tokens = t.size(0), heads = t.size(1), dim = t.size(2);
    TORCH_CHECK_VALUE((dim == 1 || t.stride(2) == 1) && (heads == 1 || t.stride(1) == dim), name,
                      ": the heads of a token must be contiguous, got strides ", t.strides());
    *stride = tokens > 1 ? t.stride(0) : heads * dim;
    return t.data_ptr();
}

// There is no backward pass: where a graph is recorded, a result outside it would drop gradients in silence.
struct Named {
    const char *name;
    const at::Tensor *t;
};
void no_gradients(std::initializer_list<Named> all)
{
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

int32_t type_code(at::ScalarType t)
{
    TORCH_CHECK_VALUE(t == at::kFloat || t == at::kBFloat16 || t == at::kHalf, "expected float32, bfloat16 or float16, got ", t);
    return t == at::kFloat ? ATTN_DT_F32 : t == at::kBFloat16 ? ATTN_DT_BF16 : ATTN_DT_F16;
}

// The shape of the layer and the caches' addresses; q is [tokens, heads, dim].
attn_shape_t layer(const at::Tensor &q, const at::Tensor &k_cache, const at::Tensor &v_cache, int device, void **k, void **v)
{
    TORCH_CHECK_VALUE(q.dim() == 3, "q: expected [tokens, heads, head_dim], got ", q.sizes());
    TORCH_CHECK_VALUE(k_cache.dim() == 4, "k_cache: expected [n_blocks, n_kv_heads, block_size, head_dim], got ", k_cache.sizes());
    const at::ScalarType type = q.scalar_type();
    attn_shape_t s;
    s.io_dtype = type_code(type);
    *k = address("k_cache", k_cache, {-1, -1, -1, -1}, type, device);
    *v = address("v_cache", v_cache, {k_cache.size(0), k_cache.size(1), k_cache.size(2), k_cache.size(3)}, type, device);
    const int64_t most = 0x7fffffff;
    TORCH_CHECK_VALUE(q.size(1) <= most && k_cache.size(0) <= most && k_cache.size(1) <= most && k_cache.size(2) <= most && k_cache.size(3) <= most,
                      "a size does not fit 32 bits");
    s.n_q_heads = (int32_t)q.size(1);
    s.n_kv_heads = (int32_t)k_cache.size(1);
    s.block_size = (int32_t)k_cache.size(2);
    s.head_dim = (int32_t)k_cache.size(3);
    return s;
}

int32_t int32_of(PyObject *o, const char *name)
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

// (block_size, total_tokens, cu_seqlens, cached_lens, table, free_blocks, n_free, shared_tail | None, in_place)
PyObject *assign_blocks(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 9);
    const int32_t block_size = int32_of(args[0], "block_size");
    const long long total = PyLong_AsLongLong(args[1]);
    if (total == -1 && PyErr_Occurred())
        throw python_error();
    TORCH_CHECK_VALUE(total >= 0, "total_tokens must not be negative");
    const at::Tensor &cu = tensor(args[2], "cu_seqlens"), &cached = tensor(args[3], "cached_lens"), &table = tensor(args[4], "table"),
                     &free_blocks = tensor(args[5], "free_blocks"), &n_free = tensor(args[6], "n_free");
    const int device = on_current_device(cu);
    const int64_t batch = cu.numel() - 1;
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device), *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device);
    const int32_t *table_at = address<int32_t>("table", table, {batch, -1}, at::kInt, device);
    const int32_t *free_at = address<int32_t>("free_blocks", free_blocks, {-1}, at::kInt, device), *n_free_at = address<int32_t>("n_free", n_free, {1}, at::kInt, device);
    const int32_t *shared_at = args[7] == Py_None ? nullptr : address<int32_t>("shared_tail", tensor(args[7], "shared_tail"), {batch}, at::kInt, device);
    const int in_place = PyObject_IsTrue(args[8]);
    if (in_place < 0)
        throw python_error();
    const at::TensorOptions ints = table.options();
    const at::Tensor out = in_place ? table : at::empty(table.sizes(), ints), slots = at::empty({total}, ints.dtype(at::kLong)),
                     positions = at::empty({total}, ints), copies = at::empty({batch, 4}, ints), counts = at::empty({2}, ints);
    check(attn_assign_blocks(size32(batch, "batch"), block_size, size32(table.size(1), "the table's width"), total, cu_at, cached_at, shared_at, table_at,
                             static_cast<int32_t *>(out.data_ptr()), free_at, n_free_at, size32(free_blocks.numel(), "free_blocks"),
                             static_cast<int64_t *>(slots.data_ptr()), static_cast<int32_t *>(positions.data_ptr()),
                             static_cast<int32_t *>(copies.data_ptr()), static_cast<int32_t *>(counts.data_ptr()), stream(device)));
    if (in_place)
        written(table);
    PyObject *r = PyTuple_New(5);
    if (!r)
        throw python_error();
    const at::Tensor *all[5] = {&out, &slots, &positions, &copies, &counts};
    for (int i = 0; i < 5; ++i)
        PyTuple_SET_ITEM(r, i, THPVariable_Wrap(*all[i]));
    return r;
    END_HANDLE_TH_ERRORS
}

// (q, k, v, positions | None, slots, rotary | None, k_cache, v_cache, interleaved, copies | None, q_out | None)
PyObject *rope_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 11);
    const at::Tensor &q = tensor(args[0], "q"), &k = tensor(args[1], "k"), &v = tensor(args[2], "v"), &slots = tensor(args[4], "slots"),
                     &k_cache = tensor(args[6], "k_cache"), &v_cache = tensor(args[7], "v_cache");
    no_gradients({{"q", &q}, {"k", &k}, {"v", &v}, {"k_cache", &k_cache}, {"v_cache", &v_cache}});
    if (args[5] != Py_None)
        no_gradients({{"rotary", &tensor(args[5], "rotary")}});
    if (args[10] != Py_None)
        no_gradients({{"q_out", &tensor(args[10], "q_out")}});
    const int device = on_current_device(q);
    const at::ScalarType type = q.scalar_type();
    void *k_to, *v_to;
    const attn_shape_t s = layer(q, k_cache, v_cache, device, &k_to, &v_to);
    const int64_t T = q.size(0);
    int64_t q_stride, k_stride, v_stride;
    const void *q_at = rows("q", q, {T, s.n_q_heads, s.head_dim}, type, device, &q_stride);
    const void *k_at = rows("k", k, {T, s.n_kv_heads, s.head_dim}, type, device, &k_stride);
    const void *v_at = rows("v", v, {T, s.n_kv_heads, s.head_dim}, type, device, &v_stride);
    const int64_t *slots_at = address<int64_t>("slots", slots, {T}, at::kLong, device);
    const int32_t *positions_at = nullptr, *copies_at = nullptr;
    const float *rotary_at = nullptr;
    int32_t most = 0, dim = 0, batch = 0;
    if (args[5] != Py_None) {
        const at::Tensor &rotary = tensor(args[5], "rotary");
        rotary_at = address<float>("rotary", rotary, {-1, 2, -1}, at::kFloat, device);
        most = size32(rotary.size(0), "rotary");
        dim = size32(2 * rotary.size(2), "rotary");
        positions_at = address<int32_t>("positions", tensor(args[3], "positions"), {T}, at::kInt, device);
    }
    const int interleaved = PyObject_IsTrue(args[8]);
    if (interleaved < 0)
        throw python_error();
    if (args[9] != Py_None) {
        const at::Tensor &copies = tensor(args[9], "copies");
        copies_at = address<int32_t>("copies", copies, {-1, 4}, at::kInt, device);
        batch = size32(copies.size(0), "copies");
    }
    const at::Tensor out = args[10] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(args[10], "q_out");
    void *out_at = address("q_out", out, {T, s.n_q_heads, s.head_dim}, type, device);
    check(attn_rope_append(&s, T, batch, size32(k_cache.size(0), "n_blocks"), q_at, q_stride, k_at, k_stride, v_at, v_stride, positions_at, slots_at,
                           rotary_at, most, dim, interleaved, copies_at, out_at, k_to, v_to, stream(device)));
    written(k_cache);
    written(v_cache);
    if (args[10] != Py_None)
        written(out);
    return THPVariable_Wrap(out);
    END_HANDLE_TH_ERRORS
}

// (q, k_cache, v_cache, table, cu_seqlens, cached_lens, scale | None, window, sinks, max_new, out | None, return_lse)
PyObject *attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 12);
    const at::Tensor &q = tensor(args[0], "q"), &k_cache = tensor(args[1], "k_cache"), &v_cache = tensor(args[2], "v_cache"), &table = tensor(args[3], "table"),
                     &cu = tensor(args[4], "cu_seqlens"), &cached = tensor(args[5], "cached_lens");
    no_gradients({{"q", &q}, {"k_cache", &k_cache}, {"v_cache", &v_cache}});
    if (args[10] != Py_None)
        no_gradients({{"out", &tensor(args[10], "out")}});
    const int device = on_current_device(q);
    const at::ScalarType type = q.scalar_type();
    void *k_at, *v_at;
    const attn_shape_t s = layer(q, k_cache, v_cache, device, &k_at, &v_at);
    const int64_t T = q.size(0), batch = cu.numel() - 1;
    int64_t q_stride, out_stride;
    const void *q_at = rows("q", q, {T, s.n_q_heads, s.head_dim}, type, device, &q_stride);
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device);
    const int32_t *table_at = address<int32_t>("table", table, {batch, -1}, at::kInt, device), *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device);
    const double given = args[6] == Py_None ? 0.0 : PyFloat_AsDouble(args[6]);
    if (given == -1.0 && PyErr_Occurred())
        throw python_error();
    const float scale = args[6] == Py_None ? (float)(1.0 / std::sqrt((double)s.head_dim)) : (float)given;
    const int32_t window = int32_of(args[7], "window"), sinks = int32_of(args[8], "sinks"), max_new = int32_of(args[9], "max_new");
    const int want_lse = PyObject_IsTrue(args[11]);
    if (want_lse < 0)
        throw python_error();
    size_t need = 0;
    check(attn_workspace_bytes(&s, size32(batch, "batch"), T, max_new, &need));
    const at::Tensor out = args[10] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(args[10], "out");
    void *out_at = rows("out", out, {T, s.n_q_heads, s.head_dim}, type, device, &out_stride);
    at::Tensor lse, workspace;
    if (want_lse)
        lse = at::empty({T, s.n_q_heads}, q.options().dtype(at::kFloat));
    if (need)
        workspace = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
    check(attn_attend(&s, (int32_t)batch, T, size32(k_cache.size(0), "n_blocks"), size32(table.size(1), "the table's width"), q_at, q_stride, k_at, v_at,
                      table_at, cu_at, cached_at, scale, window, sinks, max_new, out_at, out_stride, want_lse ? static_cast<float *>(lse.data_ptr()) : nullptr,
                      need ? workspace.data_ptr() : nullptr, need, stream(device)));
    if (args[10] != Py_None)
        written(out);
    if (!want_lse)
        return THPVariable_Wrap(out);
    PyObject *r = PyTuple_New(2);
    if (!r)
        throw python_error();
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(lse));
    return r;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error_class(PyObject *, PyObject *c)
{
    Py_INCREF(c);
    Py_XDECREF(g_error_class);
    g_error_class = c;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"assign_blocks", (PyCFunction)(void (*)(void))assign_blocks, METH_FASTCALL, nullptr},
    {"rope_append", (PyCFunction)(void (*)(void))rope_append, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attn_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attn_binding() { return PyModule_Create(&module); }
