/*
 * attn_cache.h -- C ABI of the attention layers of a hybrid model behind the
 * prefix cache, on MI355X (gfx950).
 *
 * A hybrid model has a few attention layers between its SSM layers (Section
 * 5.1, "Models"); a prefix-cache hit skips the prefill of both kinds.  What
 * the SSM layers resume from is a state (ssm_prefill.h); what the attention
 * layers resume from is the keys and values of the prefix (Section 2.1), kept
 * here in a paged cache: blocks of block_size tokens, named by the rows of a
 * block table.  Three operators, called one after the other:
 *
 *   attn_assign_blocks  once per step: blocks for the new tokens of every
 *                       request, their slots and positions
 *   attn_rope_append    once per layer: rotary positions on q and k, k and v
 *                       into the cache
 *   attn_attend         once per layer: attention of the new tokens over the
 *                       cache
 *
 * All three read the requests' lengths from device memory and only enqueue:
 * nothing here allocates, copies to the host, synchronises, or depends on
 * lengths that the host would have to know, so a step can be captured into a
 * graph and replayed while the lengths grow.
 *
 * Sequence b of a packed batch has cached_lens[b] tokens in the cache and
 * brings n_b = cu_seqlens[b+1] - cu_seqlens[b] new ones; token i of them has
 * position cached_lens[b] + i.  Its key at position j lies in block
 * table[b, j / block_size], row j % block_size.  cu_seqlens[batch] may be less
 * than total_tokens (a captured step with room for more): the tokens behind it
 * belong to no sequence, get the slot -1 and position 0, and their rows of the
 * attention's results are not written.  The caches of a layer are
 *
 *   k_cache, v_cache  [n_blocks, n_kv_heads, block_size, head_dim]  io_dtype
 *
 * "device" pointers are HIP device pointers on the current device; all tensors
 * are row-major with the last index fastest.  Every entry point returns
 * ATTN_OK (0) or a negative attn_status_t; on error nothing has been enqueued
 * and attn_last_error() returns a message for the calling thread.  Nothing here
 * throws or aborts.  Device arrays of indices are checked where they are used:
 * a block id outside the cache counts as none, lengths beyond the arrays are
 * cut, and no value of them makes a kernel access memory outside its arguments.
 */
#ifndef ATTN_CACHE_H
#define ATTN_CACHE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ATTN_OK = 0,
    ATTN_ERR_INVALID_ARG = -1,       /* NULL where a pointer is required, bad sizes */
    ATTN_ERR_UNSUPPORTED_SHAPE = -4, /* shape outside what the kernels handle       */
    ATTN_ERR_WORKSPACE_TOO_SMALL = -5,
    ATTN_ERR_MISALIGNED = -6,        /* a pointer or a stride is not a multiple of 16 bytes */
    ATTN_ERR_HIP = -7                /* a HIP runtime call failed                   */
} attn_status_t;

typedef enum { ATTN_DT_F32 = 0, ATTN_DT_BF16 = 1, ATTN_DT_F16 = 2 } attn_dtype_t; /* q, k, v, the caches, out */

typedef struct {
    int32_t n_q_heads;
    int32_t n_kv_heads; /* divides n_q_heads; query head h reads key head h / (n_q_heads / n_kv_heads) */
    int32_t head_dim;   /* attn_attend: 64 or 128; attn_rope_append: a multiple of 8 up to 256 */
    int32_t block_size; /* tokens per block of the cache, a power of two up to 1024 */
    int32_t io_dtype;   /* attn_dtype_t */
} attn_shape_t;

/*
 * Blocks for the new tokens of a batch (Section 2.1: KVs grow with every
 * token), their slots and positions.  The rows of a hit are filled in by the
 * caller from the cached sequence it resumes from (Section 2.2); this call
 * extends them.  Requests are served in order; the k-th block handed out is
 * free_blocks[n_free - 1 - k].
 *
 *   cu_seqlens   [batch+1]  int32 device, from 0 to at most total_tokens
 *   cached_lens  [batch]    int32 device
 *   shared_tail  [batch]    int32 device or NULL; nonzero: the sequence's last
 *                           cached block may be read by others (the hit ends
 *                           inside a block of a cached sequence), so if that
 *                           block is not full and there are new tokens, a new
 *                           block takes its place in the row and `copies` says
 *                           which rows have to be copied
 *   table_in, table_out  [batch, max_blocks]  int32 device; may be the same
 *                           array.  Entries of cached tokens are read from
 *                           table_in; handed-out blocks go to table_out.  With
 *                           two arrays the cached entries are copied and the
 *                           rest of every row of table_out is set to -1; with
 *                           one, nothing else of a row is touched.
 *   free_blocks  [n_free]   int32 device;  n_free: int32 device, one value,
 *                           at most free_capacity
 *   slots        [total_tokens]  int64 device, out: block * block_size + row,
 *                           or -1 for a token that got no block: the free
 *                           list ran out, or its entry lies behind the end of
 *                           the table's row (no block is taken for that)
 *   positions    [total_tokens]  int32 device, out
 *   copies       [batch, 4] int32 device, out: from block, to block, rows, 0;
 *                           (-1, -1, 0, 0) where nothing is to be copied.  If the free list
 *                           ran out "to" is -1.
 *   counts       [2]        int32 device, out: blocks left on the free list,
 *                           blocks that were missing in this call, entries of
 *                           new tokens behind the end of a row among them.
 *                           Must not overlap n_free.
 *
 * batch is at most 4096.
 */
int attn_assign_blocks(int32_t batch, int32_t block_size, int32_t max_blocks, int64_t total_tokens,
                       const int32_t *cu_seqlens, const int32_t *cached_lens, const int32_t *shared_tail,
                       const int32_t *table_in, int32_t *table_out,
                       const int32_t *free_blocks, const int32_t *n_free, int32_t free_capacity,
                       int64_t *slots, int32_t *positions, int32_t *copies, int32_t *counts,
                       void *hip_stream);

/*
 * Rotary positions and the append to the cache of one layer (the KVs a request
 * adds to its prefix, Section 2.1).  The first rotary_dim values of every q
 * and k head are turned: pair i is (x[i], x[i + rotary_dim/2]), or with
 * interleaved = 1 (x[2i], x[2i+1]), and
 *
 *     (a, b) -> (a cos - b sin, b cos + a sin),   cos, sin = rotary[position, 0..1, i]
 *
 * in fp32, rounded once.  Scaling for long contexts is in the table.
 *
 *   q [T, n_q_heads, head_dim], k and v [T, n_kv_heads, head_dim]  io_dtype,
 *       device; q_stride, k_stride, v_stride: elements between tokens (the
 *       heads of a token are contiguous), rows 16-byte aligned: the three may
 *       be parts of the rows of one projection
 *   positions [T], slots [T]   as attn_assign_blocks writes them.  A token
 *       whose slot lies outside the cache (-1) is not appended.  Positions
 *       outside 0..max_positions-1 turn into NaN.  Slots of different tokens
 *       must differ.
 *   rotary    [max_positions, 2, rotary_dim/2]  fp32, device
 *   copies    [batch, 4] or NULL: the first `rows` rows of block "from" are
 *       copied to block "to" in both caches, for all heads
 *   q_out     [T, n_q_heads, head_dim]  io_dtype, contiguous; may be q itself
 *       if q is contiguous
 *
 * rotary_dim: a multiple of 16, at most head_dim; 0: nothing turns and rotary
 * and positions may be NULL.
 */
int attn_rope_append(const attn_shape_t *shape, int64_t total_tokens, int32_t batch, int32_t n_blocks,
                     const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                     const void *v, int64_t v_stride,
                     const int32_t *positions, const int64_t *slots,
                     const float *rotary, int32_t max_positions, int32_t rotary_dim, int32_t interleaved,
                     const int32_t *copies, void *q_out, void *k_cache, void *v_cache, void *hip_stream);

/*
 * Bytes of device workspace attn_attend needs for a batch of this size: partial
 * results of rows whose keys are dealt to several workgroups.  The caller
 * allocates it, 256-byte aligned; its contents mean nothing between calls.
 */
int attn_workspace_bytes(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t max_new,
                         size_t *bytes);

/*
 * Attention of the new tokens of a batch over the cache, which holds their own
 * keys and values already (attn_rope_append).  The query at position p sees the
 * key at position j if
 *
 *     j <= p   and   (window == 0  or  j > p - window  or  j < sinks)
 *
 * and table[b, j / block_size] names a block of the cache.
 *
 *     out = sum_j softmax_j(scale * q . k_j) v_j,    lse = ln sum_j exp(scale * q . k_j)
 *
 * over the keys it sees; a query that sees none gets out = 0, lse = -inf.  One
 * whose largest scaled score is minus infinity or beyond fp32 gets NaN.
 * Statistics and sums are fp32; with 16-bit types the weights are rounded to
 * the type for the product with v.
 *
 *   q, out  [T, n_q_heads, head_dim] io_dtype, device; q_stride, out_stride:
 *           elements between tokens, rows 16-byte aligned
 *   lse     [T, n_q_heads] fp32 device, or NULL
 *   scale   positive and finite
 *   max_new 0, or the largest number of new tokens of any sequence as far as
 *           the caller knows it: it decides between kernels for single tokens
 *           and for chunks and nothing else (a wrong value costs time; 0 takes
 *           a batch with no more tokens than sequences for single tokens)
 *   workspace  >= attn_workspace_bytes of the same batch, total_tokens and
 *           max_new; may be NULL if that is 0
 *
 * batch is at most 4096.  Results do not depend on the timing of the GPU; how
 * the keys of a sequence are dealt out, and with it the rounding, may depend on
 * the other sequences of the batch.
 */
int attn_attend(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks, int32_t max_blocks,
                const void *q, int64_t q_stride, const void *k_cache, const void *v_cache,
                const int32_t *table, const int32_t *cu_seqlens, const int32_t *cached_lens,
                float scale, int32_t window, int32_t sinks, int32_t max_new,
                void *out, int64_t out_stride, float *lse,
                void *workspace, size_t workspace_bytes, void *hip_stream);

/* Message of the last error on the calling thread ("" if none). */
const char *attn_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ATTN_CACHE_H */
