// Entry points of the attention operators: argument checks and launches.  Nothing here allocates or synchronises.
#include <algorithm>
#include <cmath>
#include <string>

#include "attn_common.h"

namespace {

thread_local std::string g_error;

int fail(int code, const char *msg)
{
    try {
        g_error = msg;
    } catch (...) {  // no memory for the message: the code says it
    }
    return code;
}

int hip_status(hipError_t e)
{
    if (e == hipSuccess)
        return ATTN_OK;
    return fail(ATTN_ERR_HIP, hipGetErrorString(e));
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_shape(const attn_shape_t *s)
{
    if (!s)
        return fail(ATTN_ERR_INVALID_ARG, "shape is NULL");
    if (s->n_q_heads < 1 || s->n_kv_heads < 1 || s->head_dim < 1)
        return fail(ATTN_ERR_INVALID_ARG, "head counts and head_dim must be positive");
    if (s->n_q_heads % s->n_kv_heads != 0)
        return fail(ATTN_ERR_INVALID_ARG, "n_kv_heads must divide n_q_heads");
    if (s->io_dtype != ATTN_DT_F32 && s->io_dtype != ATTN_DT_BF16 && s->io_dtype != ATTN_DT_F16)
        return fail(ATTN_ERR_INVALID_ARG, "io_dtype is not one of attn_dtype_t");
    if (s->block_size < 1 || s->block_size > 1024 || (s->block_size & (s->block_size - 1)) != 0)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "block_size must be a power of two up to 1024");
    if (s->n_q_heads > 1024)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "at most 1024 query heads");
    return ATTN_OK;
}

int check_batch(int32_t batch, int64_t total_tokens)
{
    if (batch < 0 || total_tokens < 0)
        return fail(ATTN_ERR_INVALID_ARG, "batch and total_tokens must not be negative");
    if (batch > kMaxBatch)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "at most 4096 sequences per call");
    if (total_tokens > 0x3fffffff)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "at most 2^30 - 1 tokens per call");
    return ATTN_OK;
}

int check_cache(const attn_shape_t *s, int32_t n_blocks)
{
    if (n_blocks < 1)
        return fail(ATTN_ERR_INVALID_ARG, "the cache needs at least one block");
    if ((int64_t)n_blocks * s->n_kv_heads * s->block_size > 0x7fffffff)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "n_blocks * n_kv_heads * block_size must be below 2^31");
    return ATTN_OK;
}

// A row of `heads` heads every `stride` elements.
int check_rows(const attn_shape_t *s, const void *p, int64_t stride, int heads, const char *what)
{
    if (!p)
        return fail(ATTN_ERR_INVALID_ARG, what);
    const int64_t esz = s->io_dtype == ATTN_DT_F32 ? 4 : 2;
    if (stride < (int64_t)heads * s->head_dim || stride > (int64_t)1 << 40)
        return fail(ATTN_ERR_INVALID_ARG, "a token stride is shorter than the token's heads, or not a length");
    if (!aligned16(p) || stride * esz % 16 != 0)
        return fail(ATTN_ERR_MISALIGNED, "device pointers and token strides must be multiples of 16 bytes");
    return ATTN_OK;
}

int check_attend_shape(const attn_shape_t *s)
{
    const int rc = check_shape(s);
    if (rc != ATTN_OK)
        return rc;
    if (s->head_dim != 64 && s->head_dim != 128)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "attn_attend handles a head_dim of 64 or 128");
    return ATTN_OK;
}

int check_attend_batch(const attn_shape_t *s, int32_t batch, int64_t total_tokens)
{
    const int rc = check_batch(batch, total_tokens);
    if (rc != ATTN_OK)
        return rc;
    if (total_tokens * (s->n_q_heads / s->n_kv_heads) > 0x3fffffff)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "total_tokens times the heads of a group must be below 2^30");
    return ATTN_OK;
}

int check_tree_words(int32_t words)
{
    if (words < 1 || words > kMostTreeWords)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "a tree has 1 to 32 words of bits, up to 1024 tokens");
    return ATTN_OK;
}

constexpr int kMostCaches = 256;

}  // namespace

extern "C" const char *attn_last_error(void) { return g_error.c_str(); }

extern "C" int attn_assign_blocks(int32_t batch, int32_t block_size, int32_t max_blocks, int64_t total_tokens,
                                  const int32_t *cu_seqlens, const int32_t *cached_lens, const int32_t *shared_tail,
                                  const int32_t *table_in, int32_t *table_out, const int32_t *free_blocks,
                                  const int32_t *n_free, int32_t free_capacity, int64_t *slots, int32_t *positions,
                                  int32_t *copies, int32_t *counts, void *hip_stream)
{
    int rc = check_batch(batch, total_tokens);
    if (rc != ATTN_OK)
        return rc;
    if (block_size < 1 || block_size > 1024 || (block_size & (block_size - 1)) != 0)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "block_size must be a power of two up to 1024");
    if (max_blocks < 1 || free_capacity < 0)
        return fail(ATTN_ERR_INVALID_ARG, "max_blocks must be positive, free_capacity not negative");
    if (batch == 0)
        return total_tokens == 0 ? ATTN_OK : fail(ATTN_ERR_INVALID_ARG, "tokens without sequences");
    if (!cu_seqlens || !cached_lens || !table_in || !table_out || !n_free || !copies || !counts)
        return fail(ATTN_ERR_INVALID_ARG, "a required pointer is NULL");
    if (free_capacity > 0 && !free_blocks)
        return fail(ATTN_ERR_INVALID_ARG, "free_blocks is NULL");
    if (total_tokens > 0 && (!slots || !positions))
        return fail(ATTN_ERR_INVALID_ARG, "slots and positions are required where there are tokens");
    if (n_free >= counts && n_free < counts + 2)
        return fail(ATTN_ERR_INVALID_ARG, "counts must not overlap n_free: every workgroup reads n_free");
    return hip_status(launch_attn_assign(batch, __builtin_ctz((unsigned)block_size), max_blocks, total_tokens, cu_seqlens,
                                         cached_lens, shared_tail, table_in, table_out, free_blocks, n_free, free_capacity,
                                         slots, positions, copies, counts, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int attn_rope_append(const attn_shape_t *shape, int64_t total_tokens, int32_t batch, int32_t n_blocks,
                                const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v,
                                int64_t v_stride, const int32_t *positions, const int64_t *slots, const float *rotary,
                                int32_t max_positions, int32_t rotary_dim, int32_t interleaved, const int32_t *copies,
                                void *q_out, void *k_cache, void *v_cache, void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == ATTN_OK)
        rc = check_batch(batch, total_tokens);
    if (rc == ATTN_OK)
        rc = check_cache(shape, n_blocks);
    if (rc != ATTN_OK)
        return rc;
    const attn_shape_t &s = *shape;
    if (s.head_dim % 8 != 0 || s.head_dim > 256)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "attn_rope_append handles a head_dim that is a multiple of 8 up to 256");
    if (rotary_dim < 0 || rotary_dim > s.head_dim || rotary_dim % 16 != 0)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "rotary_dim must be a multiple of 16 up to head_dim");
    if (interleaved != 0 && interleaved != 1)
        return fail(ATTN_ERR_INVALID_ARG, "interleaved is 0 or 1");
    if (!k_cache || !v_cache)
        return fail(ATTN_ERR_INVALID_ARG, "k_cache or v_cache is NULL");
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(rotary) || !aligned16(q_out))
        return fail(ATTN_ERR_MISALIGNED, "device pointers must be 16-byte aligned");
    if (total_tokens > 0) {
        rc = check_rows(shape, q, q_stride, s.n_q_heads, "q is NULL");
        if (rc == ATTN_OK)
            rc = check_rows(shape, k, k_stride, s.n_kv_heads, "k is NULL");
        if (rc == ATTN_OK)
            rc = check_rows(shape, v, v_stride, s.n_kv_heads, "v is NULL");
        if (rc != ATTN_OK)
            return rc;
        if (!q_out || !slots)
            return fail(ATTN_ERR_INVALID_ARG, "q_out or slots is NULL");
        if (q_out == q && q_stride != (int64_t)s.n_q_heads * s.head_dim)
            return fail(ATTN_ERR_INVALID_ARG, "q_out may be q only if q is contiguous");
        if (rotary_dim > 0 && (!positions || !rotary || max_positions < 1))
            return fail(ATTN_ERR_INVALID_ARG, "positions and a rotary table are required where something turns");
    }
    return hip_status(launch_attn_rope(s, total_tokens, batch, n_blocks, q, q_stride, k, k_stride, v, v_stride, positions,
                                       slots, rotary, max_positions, rotary_dim, interleaved != 0, copies, q_out, k_cache,
                                       v_cache, static_cast<hipStream_t>(hip_stream)));
}

static int attend_workspace(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t max_new, bool trees, size_t *bytes)
{
    int rc = check_attend_shape(shape);
    if (rc == ATTN_OK)
        rc = check_attend_batch(shape, batch, total_tokens);
    if (rc != ATTN_OK)
        return rc;
    if (!bytes || max_new < 0)
        return fail(ATTN_ERR_INVALID_ARG, "bytes is NULL or max_new negative");
    *bytes = trees ? attn_attend_tree_workspace(*shape, batch, total_tokens, max_new) : attn_attend_workspace(*shape, batch, total_tokens, max_new);
    return ATTN_OK;
}

extern "C" int attn_workspace_bytes(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t max_new,
                                    size_t *bytes)
{
    return attend_workspace(shape, batch, total_tokens, max_new, false, bytes);
}

extern "C" int attn_tree_workspace_bytes(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t max_new,
                                         size_t *bytes)
{
    return attend_workspace(shape, batch, total_tokens, max_new, true, bytes);
}

static int attend(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks, int32_t max_blocks,
                  const void *q, int64_t q_stride, const void *k_cache, const void *v_cache, const int32_t *table,
                  const int32_t *cu_seqlens, const int32_t *cached_lens, const AttnTrees &trees, float scale, int32_t window,
                  int32_t sinks, int32_t max_new, void *out, int64_t out_stride, float *lse, void *workspace,
                  size_t workspace_bytes, void *hip_stream)
{
    int rc = check_attend_shape(shape);
    if (rc == ATTN_OK)
        rc = check_attend_batch(shape, batch, total_tokens);
    if (rc == ATTN_OK)
        rc = check_cache(shape, n_blocks);
    if (rc != ATTN_OK)
        return rc;
    if (max_blocks < 1 || window < 0 || sinks < 0 || max_new < 0)
        return fail(ATTN_ERR_INVALID_ARG, "max_blocks must be positive; window, sinks and max_new must not be negative");
    if (!(scale > 0.f) || !std::isfinite(scale) || !std::isnormal(scale * kLog2e))
        return fail(ATTN_ERR_INVALID_ARG, "scale must be positive and finite");
    if (total_tokens == 0)
        return ATTN_OK;
    if (batch == 0)
        return fail(ATTN_ERR_INVALID_ARG, "tokens without sequences");
    if (!k_cache || !v_cache || !table || !cu_seqlens || !cached_lens)
        return fail(ATTN_ERR_INVALID_ARG, "a required pointer is NULL");
    rc = check_rows(shape, q, q_stride, shape->n_q_heads, "q is NULL");
    if (rc == ATTN_OK)
        rc = check_rows(shape, out, out_stride, shape->n_q_heads, "out is NULL");
    if (rc != ATTN_OK)
        return rc;
    if (!aligned16(k_cache) || !aligned16(v_cache))
        return fail(ATTN_ERR_MISALIGNED, "device pointers must be 16-byte aligned");
    const bool is_tree = trees.words > 0;
    const size_t need = is_tree ? attn_attend_tree_workspace(*shape, batch, total_tokens, max_new) : attn_attend_workspace(*shape, batch, total_tokens, max_new);
    if (need) {
        if (!workspace || workspace_bytes < need)
            return fail(ATTN_ERR_WORKSPACE_TOO_SMALL, "workspace is NULL or smaller than attn_workspace_bytes");
        if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
            return fail(ATTN_ERR_MISALIGNED, "workspace is not 256-byte aligned");
    }
    if (is_tree)
        return hip_status(launch_attn_attend_tree(*shape, batch, total_tokens, n_blocks, max_blocks, q, q_stride, k_cache, v_cache,
                                                  table, cu_seqlens, cached_lens, scale, window, sinks, max_new, out, out_stride,
                                                  lse, workspace, static_cast<hipStream_t>(hip_stream), trees));
    return hip_status(launch_attn_attend(*shape, batch, total_tokens, n_blocks, max_blocks, q, q_stride, k_cache, v_cache,
                                         table, cu_seqlens, cached_lens, scale, window, sinks, max_new, out, out_stride, lse,
                                         workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int attn_attend(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks,
                           int32_t max_blocks, const void *q, int64_t q_stride, const void *k_cache, const void *v_cache,
                           const int32_t *table, const int32_t *cu_seqlens, const int32_t *cached_lens, float scale,
                           int32_t window, int32_t sinks, int32_t max_new, void *out, int64_t out_stride, float *lse,
                           void *workspace, size_t workspace_bytes, void *hip_stream)
{
    return attend(shape, batch, total_tokens, n_blocks, max_blocks, q, q_stride, k_cache, v_cache, table, cu_seqlens, cached_lens,
                  AttnTrees(), scale, window, sinks, max_new, out, out_stride, lse, workspace, workspace_bytes, hip_stream);
}

extern "C" int attn_attend_tree(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks,
                                int32_t max_blocks, const void *q, int64_t q_stride, const void *k_cache, const void *v_cache,
                                const int32_t *table, const int32_t *cu_seqlens, const int32_t *cached_lens,
                                const int32_t *positions, const int32_t *seen, int32_t words, float scale, int32_t window,
                                int32_t sinks, int32_t max_new, void *out, int64_t out_stride, float *lse, void *workspace,
                                size_t workspace_bytes, void *hip_stream)
{
    int rc = check_tree_words(words);
    if (rc == ATTN_OK && total_tokens > 0 && (!positions || !seen))
        rc = fail(ATTN_ERR_INVALID_ARG, "positions or seen is NULL");
    if (rc != ATTN_OK)
        return rc;
    AttnTrees trees;
    trees.positions = positions, trees.seen = seen, trees.words = words;
    return attend(shape, batch, total_tokens, n_blocks, max_blocks, q, q_stride, k_cache, v_cache, table, cu_seqlens, cached_lens,
                  trees, scale, window, sinks, max_new, out, out_stride, lse, workspace, workspace_bytes, hip_stream);
}

extern "C" int attn_draft_tree(int32_t batch, int64_t total_tokens, int32_t words, const int32_t *parents,
                               const int32_t *cu_seqlens, const int32_t *cached_lens, int32_t window, int32_t sinks,
                               int32_t *positions, int32_t *seen, void *hip_stream)
{
    int rc = check_batch(batch, total_tokens);
    if (rc == ATTN_OK)
        rc = check_tree_words(words);
    if (rc != ATTN_OK)
        return rc;
    if (window < 0 || sinks < 0)
        return fail(ATTN_ERR_INVALID_ARG, "window and sinks must not be negative");
    if (total_tokens == 0)
        return ATTN_OK;
    if (batch == 0)
        return fail(ATTN_ERR_INVALID_ARG, "tokens without sequences");
    if (!parents || !cu_seqlens || !cached_lens || !positions || !seen)
        return fail(ATTN_ERR_INVALID_ARG, "a required pointer is NULL");
    return hip_status(launch_attn_draft_tree(batch, total_tokens, words, parents, cu_seqlens, cached_lens, window, sinks, positions,
                                             seen, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int attn_accept_path(int32_t batch, int32_t block_size, int32_t max_blocks, int64_t total_tokens,
                                const int32_t *tokens, const int32_t *parents, const int32_t *choices,
                                const int32_t *cu_seqlens, const int32_t *cached_lens, int32_t *path, int32_t *counts,
                                int32_t *next_tokens, int32_t *kept_lens, const int32_t *table, int32_t *free_blocks,
                                int32_t free_capacity, const int32_t *n_free, int32_t *n_free_out, void *hip_stream)
{
    const int rc = check_batch(batch, total_tokens);
    if (rc != ATTN_OK)
        return rc;
    if (batch == 0)
        return total_tokens == 0 ? ATTN_OK : fail(ATTN_ERR_INVALID_ARG, "tokens without sequences");
    if (!cu_seqlens || !cached_lens || !counts || !next_tokens || !kept_lens)
        return fail(ATTN_ERR_INVALID_ARG, "a required pointer is NULL");
    if (total_tokens > 0 && (!tokens || !parents || !choices || !path))
        return fail(ATTN_ERR_INVALID_ARG, "tokens, parents, choices and path are required where there are tokens");
    int log2_bs = 0;
    if (table) {
        if (block_size < 1 || block_size > 1024 || (block_size & (block_size - 1)) != 0)
            return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "block_size must be a power of two up to 1024");
        if (max_blocks < 1 || free_capacity < 0)
            return fail(ATTN_ERR_INVALID_ARG, "max_blocks must be positive, free_capacity not negative");
        if (!n_free || !n_free_out || (free_capacity > 0 && !free_blocks))
            return fail(ATTN_ERR_INVALID_ARG, "free_blocks, n_free and n_free_out are required with a table");
        if (n_free == n_free_out)
            return fail(ATTN_ERR_INVALID_ARG, "n_free_out must not be n_free: all threads read n_free");
        log2_bs = __builtin_ctz((unsigned)block_size);
    }
    return hip_status(launch_attn_accept(batch, log2_bs, max_blocks, total_tokens, tokens, parents, choices, cu_seqlens, cached_lens,
                                         table, free_blocks, n_free, free_capacity, path, counts, next_tokens, kept_lens,
                                         n_free_out, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int attn_keep_path(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks,
                              int32_t max_blocks, int32_t n_caches, void *const *caches, const int32_t *table,
                              const int32_t *cu_seqlens, const int32_t *cached_lens, const int32_t *path, void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == ATTN_OK)
        rc = check_batch(batch, total_tokens);
    if (rc == ATTN_OK)
        rc = check_cache(shape, n_blocks);
    if (rc != ATTN_OK)
        return rc;
    const attn_shape_t &s = *shape;
    if (s.head_dim % 8 != 0 || s.head_dim > 256)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "attn_keep_path handles a head_dim that is a multiple of 8 up to 256");
    if (n_caches < 0 || n_caches > kMostCaches)
        return fail(ATTN_ERR_UNSUPPORTED_SHAPE, "at most 256 caches per call");
    if (max_blocks < 1 || (n_caches > 0 && !caches))
        return fail(ATTN_ERR_INVALID_ARG, "max_blocks must be positive, caches must not be NULL");
    const unsigned char *at[kMostCaches];
    for (int c = 0; c < n_caches; ++c) {
        if (!caches[c])
            return fail(ATTN_ERR_INVALID_ARG, "a cache is NULL");
        if (!aligned16(caches[c]))
            return fail(ATTN_ERR_MISALIGNED, "device pointers must be 16-byte aligned");
        at[c] = static_cast<const unsigned char *>(caches[c]);
    }
    // rows that move in two caches at once would be overwritten before they have been read
    const int64_t bytes = (int64_t)n_blocks * s.n_kv_heads * s.block_size * s.head_dim * (s.io_dtype == ATTN_DT_F32 ? 4 : 2);
    std::sort(at, at + n_caches);
    for (int c = 1; c < n_caches; ++c)
        if (at[c] - at[c - 1] < bytes)
            return fail(ATTN_ERR_INVALID_ARG, "two caches overlap");
    if (total_tokens == 0 || n_caches == 0)
        return ATTN_OK;
    if (batch == 0)
        return fail(ATTN_ERR_INVALID_ARG, "tokens without sequences");
    if (!table || !cu_seqlens || !cached_lens || !path)
        return fail(ATTN_ERR_INVALID_ARG, "a required pointer is NULL");
    return hip_status(launch_attn_keep(s, batch, total_tokens, n_blocks, max_blocks, n_caches, caches, table, cu_seqlens,
                                       cached_lens, path, static_cast<hipStream_t>(hip_stream)));
}
