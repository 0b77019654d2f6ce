// CPython binding of the attention operators over their C ABI (include/attn_cache.h, include/attn_tree.h): checks of tensors, outputs and workspace
// from torch's allocator, the current stream.  A decode step of a layer is a few microseconds of GPU work, and the same steps
// written in Python with ctypes took longer than that (append 10.7 us and attention 10.0 us per call in front of the launches).
#include "torch_binding.h"

#include "attn_tree.h"

namespace {

void check(int status) { check(status, attn_last_error); }

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

// `trees`: positions and seen, behind cached_lens; then scale | None, window, sinks, max_new, out | None, return_lse
PyObject *attend_with(PyObject *const *args, bool trees)
{
    const at::Tensor &q = tensor(args[0], "q"), &k_cache = tensor(args[1], "k_cache"), &v_cache = tensor(args[2], "v_cache"), &table = tensor(args[3], "table"),
                     &cu = tensor(args[4], "cu_seqlens"), &cached = tensor(args[5], "cached_lens");
    PyObject *const *const more = args + (trees ? 8 : 6);
    no_gradients({{"q", &q}, {"k_cache", &k_cache}, {"v_cache", &v_cache}});
    if (more[4] != Py_None)
        no_gradients({{"out", &tensor(more[4], "out")}});
    const int device = on_current_device(q);
    const at::ScalarType type = q.scalar_type();
    void *k_at, *v_at;
    const attn_shape_t s = layer(q, k_cache, v_cache, device, &k_at, &v_at);
    const int64_t T = q.size(0), batch = cu.numel() - 1;
    int64_t q_stride, out_stride;
    const void *q_at = rows("q", q, {T, s.n_q_heads, s.head_dim}, type, device, &q_stride);
    const int32_t *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device);
    const int32_t *table_at = address<int32_t>("table", table, {batch, -1}, at::kInt, device), *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device);
    const int32_t *positions_at = nullptr, *seen_at = nullptr;
    int32_t words = 0;
    if (trees) {
        const at::Tensor &seen = tensor(args[7], "seen");
        positions_at = address<int32_t>("positions", tensor(args[6], "positions"), {T}, at::kInt, device);
        seen_at = address<int32_t>("seen", seen, {T, -1}, at::kInt, device);
        words = size32(seen.size(1), "seen");
    }
    const double given = more[0] == Py_None ? 0.0 : PyFloat_AsDouble(more[0]);
    if (given == -1.0 && PyErr_Occurred())
        throw python_error();
    const float scale = more[0] == Py_None ? (float)(1.0 / std::sqrt((double)s.head_dim)) : (float)given;
    const int32_t window = int32_of(more[1], "window"), sinks = int32_of(more[2], "sinks"), max_new = int32_of(more[3], "max_new");
    const int want_lse = PyObject_IsTrue(more[5]);
    if (want_lse < 0)
        throw python_error();
    size_t need = 0;
    check((trees ? attn_tree_workspace_bytes : attn_workspace_bytes)(&s, size32(batch, "batch"), T, max_new, &need));
    const at::Tensor out = more[4] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(more[4], "out");
    void *out_at = rows("out", out, {T, s.n_q_heads, s.head_dim}, type, device, &out_stride);
    at::Tensor lse, workspace;
    if (want_lse)
        lse = at::empty({T, s.n_q_heads}, q.options().dtype(at::kFloat));
    if (need)
        workspace = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
    const int32_t n_blocks = size32(k_cache.size(0), "n_blocks"), max_blocks = size32(table.size(1), "the table's width");
    float *const lse_at = want_lse ? static_cast<float *>(lse.data_ptr()) : nullptr;
    void *const workspace_at = need ? workspace.data_ptr() : nullptr;
    check(trees ? attn_attend_tree(&s, (int32_t)batch, T, n_blocks, max_blocks, q_at, q_stride, k_at, v_at, table_at, cu_at, cached_at, positions_at, seen_at,
                                   words, scale, window, sinks, max_new, out_at, out_stride, lse_at, workspace_at, need, stream(device))
                : attn_attend(&s, (int32_t)batch, T, n_blocks, max_blocks, q_at, q_stride, k_at, v_at, table_at, cu_at, cached_at, scale, window, sinks,
                              max_new, out_at, out_stride, lse_at, workspace_at, need, stream(device)));
    if (more[4] != Py_None)
        written(out);
    if (!want_lse)
        return THPVariable_Wrap(out);
    PyObject *r = PyTuple_New(2);
    if (!r)
        throw python_error();
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(out));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(lse));
    return r;
}

// (q, k_cache, v_cache, table, cu_seqlens, cached_lens, scale | None, window, sinks, max_new, out | None, return_lse)
PyObject *attend(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 12);
    return attend_with(args, false);
    END_HANDLE_TH_ERRORS
}

// (q, k_cache, v_cache, table, cu_seqlens, cached_lens, positions, seen, scale | None, window, sinks, max_new, out | None, return_lse)
PyObject *attend_tree(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 14);
    return attend_with(args, true);
    END_HANDLE_TH_ERRORS
}

// (parents, cu_seqlens, cached_lens, max_new, window, sinks)
PyObject *draft_tree(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 6);
    const at::Tensor &parents = tensor(args[0], "parents"), &cu = tensor(args[1], "cu_seqlens"), &cached = tensor(args[2], "cached_lens");
    const int device = on_current_device(parents);
    const int64_t T = parents.numel(), batch = cu.numel() - 1;
    const int32_t *parents_at = address<int32_t>("parents", parents, {-1}, at::kInt, device), *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device);
    const int32_t *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device);
    const int32_t max_new = int32_of(args[3], "max_new"), window = int32_of(args[4], "window"), sinks = int32_of(args[5], "sinks");
    TORCH_CHECK_VALUE(max_new >= 1 && max_new <= 1024, "max_new: a tree has 1 to 1024 tokens, got ", max_new);
    const int32_t words = (max_new + 31) / 32;
    const at::Tensor positions = at::empty({T}, parents.options()), seen = at::empty({T, words}, parents.options());
    check(attn_draft_tree(size32(batch, "batch"), T, words, parents_at, cu_at, cached_at, window, sinks, static_cast<int32_t *>(positions.data_ptr()),
                          static_cast<int32_t *>(seen.data_ptr()), stream(device)));
    return tuple_of({&positions, &seen});
    END_HANDLE_TH_ERRORS
}

// (tokens, parents, choices, cu_seqlens, cached_lens, block_size, table | None, free_blocks | None, n_free | None)
PyObject *accept_path(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 9);
    const at::Tensor &tokens = tensor(args[0], "tokens"), &parents = tensor(args[1], "parents"), &choices = tensor(args[2], "choices"),
                     &cu = tensor(args[3], "cu_seqlens"), &cached = tensor(args[4], "cached_lens");
    const int device = on_current_device(tokens);
    const int64_t T = tokens.numel(), batch = cu.numel() - 1;
    const int32_t *tokens_at = address<int32_t>("tokens", tokens, {-1}, at::kInt, device), *parents_at = address<int32_t>("parents", parents, {T}, at::kInt, device);
    const int32_t *choices_at = address<int32_t>("choices", choices, {T}, at::kInt, device), *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device);
    const int32_t *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device);
    const int32_t block_size = int32_of(args[5], "block_size");
    const int32_t *table_at = nullptr, *n_free_at = nullptr;
    int32_t *free_at = nullptr, max_blocks = 0, capacity = 0;
    const bool gives_back = args[6] != Py_None;
    TORCH_CHECK_VALUE(gives_back == (args[7] != Py_None) && gives_back == (args[8] != Py_None), "table, free_blocks and n_free are given together or not at all");
    if (gives_back) {
        const at::Tensor &table = tensor(args[6], "table"), &free_blocks = tensor(args[7], "free_blocks");
        table_at = address<int32_t>("table", table, {batch, -1}, at::kInt, device);
        free_at = address<int32_t>("free_blocks", free_blocks, {-1}, at::kInt, device);
        n_free_at = address<int32_t>("n_free", tensor(args[8], "n_free"), {1}, at::kInt, device);
        max_blocks = size32(table.size(1), "the table's width");
        capacity = size32(free_blocks.numel(), "free_blocks");
    }
    const at::TensorOptions ints = tokens.options();
    const at::Tensor path = at::empty({T}, ints), counts = at::empty({batch}, ints), next_tokens = at::empty({batch}, ints), kept_lens = at::empty({batch}, ints);
    at::Tensor left;
    if (gives_back)  // (nothing is enqueued for no sequences)
        left = batch > 0 ? at::empty({1}, ints) : tensor(args[8], "n_free").clamp(0, capacity);
    check(attn_accept_path(size32(batch, "batch"), block_size, max_blocks, T, tokens_at, parents_at, choices_at, cu_at, cached_at,
                           static_cast<int32_t *>(path.data_ptr()), static_cast<int32_t *>(counts.data_ptr()), static_cast<int32_t *>(next_tokens.data_ptr()),
                           static_cast<int32_t *>(kept_lens.data_ptr()), table_at, free_at, capacity, n_free_at,
                           gives_back ? static_cast<int32_t *>(left.data_ptr()) : nullptr, stream(device)));
    if (gives_back)
        written(tensor(args[7], "free_blocks"));
    return tuple_of({&path, &counts, &next_tokens, &kept_lens, &left});
    END_HANDLE_TH_ERRORS
}

// (caches, table, cu_seqlens, cached_lens, path)
PyObject *keep_path(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    arguments(n, 5);
    TORCH_CHECK_TYPE(PyList_Check(args[0]) || PyTuple_Check(args[0]), "caches: expected a list of tensors, got ", Py_TYPE(args[0])->tp_name);
    const bool list = PyList_Check(args[0]);
    const Py_ssize_t n_caches = list ? PyList_GET_SIZE(args[0]) : PyTuple_GET_SIZE(args[0]);
    TORCH_CHECK_VALUE(n_caches <= 256, "caches: at most 256 per call, got ", n_caches);
    const at::Tensor *caches[256];
    for (Py_ssize_t c = 0; c < n_caches; ++c) {
        caches[c] = &tensor(list ? PyList_GET_ITEM(args[0], c) : PyTuple_GET_ITEM(args[0], c), "caches");
        no_gradients({{"a cache", caches[c]}});
    }
    const at::Tensor &table = tensor(args[1], "table"), &cu = tensor(args[2], "cu_seqlens"), &cached = tensor(args[3], "cached_lens"), &path = tensor(args[4], "path");
    const int device = on_current_device(path);
    const int64_t T = path.numel(), batch = cu.numel() - 1;
    const int32_t *table_at = address<int32_t>("table", table, {batch, -1}, at::kInt, device), *cu_at = address<int32_t>("cu_seqlens", cu, {-1}, at::kInt, device);
    const int32_t *cached_at = address<int32_t>("cached_lens", cached, {batch}, at::kInt, device), *path_at = address<int32_t>("path", path, {-1}, at::kInt, device);
    void *at_[256];
    attn_shape_t s = {};
    int32_t n_blocks = 0;
    for (Py_ssize_t c = 0; c < n_caches; ++c) {
        const at::Tensor &x = *caches[c], &first = *caches[0];
        TORCH_CHECK_VALUE(x.dim() == 4, "caches: expected [n_blocks, n_kv_heads, block_size, head_dim], got ", x.sizes());
        at_[c] = address("caches", x, {first.size(0), first.size(1), first.size(2), first.size(3)}, first.scalar_type(), device);
    }
    if (n_caches > 0) {
        const at::Tensor &x = *caches[0];
        s.io_dtype = type_code(x.scalar_type());
        n_blocks = size32(x.size(0), "n_blocks");
        s.n_q_heads = s.n_kv_heads = size32(x.size(1), "n_kv_heads");
        s.block_size = size32(x.size(2), "block_size");
        s.head_dim = size32(x.size(3), "head_dim");
        check(attn_keep_path(&s, size32(batch, "batch"), T, n_blocks, size32(table.size(1), "the table's width"), (int32_t)n_caches, at_, table_at, cu_at,
                             cached_at, path_at, stream(device)));
        for (Py_ssize_t c = 0; c < n_caches; ++c)
            written(*caches[c]);
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"assign_blocks", (PyCFunction)(void (*)(void))assign_blocks, METH_FASTCALL, nullptr},
    {"rope_append", (PyCFunction)(void (*)(void))rope_append, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {"draft_tree", (PyCFunction)(void (*)(void))draft_tree, METH_FASTCALL, nullptr},
    {"attend_tree", (PyCFunction)(void (*)(void))attend_tree, METH_FASTCALL, nullptr},
    {"accept_path", (PyCFunction)(void (*)(void))accept_path, METH_FASTCALL, nullptr},
    {"keep_path", (PyCFunction)(void (*)(void))keep_path, METH_FASTCALL, nullptr},
    {"set_error_class", set_error_class, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attn_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attn_binding() { return PyModule_Create(&module); }
