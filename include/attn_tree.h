/*
 * attn_tree.h -- C ABI of steps that check trees of drafted tokens over the
 * paged cache of attn_cache.h, instead of adding a chain to each sequence, on
 * MI355X (gfx950).  Four operators beside those of attn_cache.h:
 *
 *   attn_draft_tree     once per step, beside attn_assign_blocks: positions of
 *                       the tokens and which of them each sees
 *   attn_attend_tree    once per layer, in the place of attn_attend
 *   attn_accept_path    once per step, behind the model: the branch that it
 *                       agrees with; blocks that are not needed are given back
 *   attn_keep_path      the branch's keys and values to where a chain has them
 *
 * What attn_cache.h says of lengths, graphs, index arrays, pointers, errors and
 * streams holds for them too; nothing that is written overlaps anything else.
 * All are in libattn_cache.so.
 */
#ifndef ATTN_TREE_H
#define ATTN_TREE_H

#include "attn_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A step whose new tokens are trees (drafts that the model checks at once).
 * New token i of a sequence, i < n_b, lies in the cache where a chain's would,
 * at row cached_lens[b] + i of its blocks (attn_assign_blocks, the slots of
 * attn_rope_append), but continues its parent: parents[t] is the index in its
 * sequence of the token in front of it, less than its own, or -1 (any other
 * value is taken for that) if only the cached ones are in front.  Token 0 is
 * as a rule the token that the step before has chosen, and all others are its
 * descendants.
 *
 * attn_draft_tree computes, once per step,
 *
 *   positions  [total_tokens]  int32: cached_lens[b] + the number of ancestors:
 *              what attn_rope_append and attn_attend_tree take
 *   seen       [total_tokens, words]  int32: bit j % 32 of word j / 32 says
 *              that the query of this token sees new token j of its sequence:
 *              itself and its ancestors; with a window those fewer than `window`
 *              positions in front of it or at a position below `sinks`
 *
 * with words = ceil(n / 32) for the longest sequence's n, 1 to 32.  New tokens
 * behind the bits are in no tree: they see nothing, their position is
 * cached_lens[b].  Tokens of no sequence get zeros.
 */
int attn_draft_tree(int32_t batch, int64_t total_tokens, int32_t words, const int32_t *parents,
                    const int32_t *cu_seqlens, const int32_t *cached_lens, int32_t window, int32_t sinks,
                    int32_t *positions, int32_t *seen, void *hip_stream);

/* As attn_workspace_bytes, for attn_attend_tree. */
int attn_tree_workspace_bytes(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t max_new,
                              size_t *bytes);

/*
 * attn_attend for such a step, with the same arguments and results, but that the
 * query of new token i sees
 *
 *   cached keys j < cached_lens[b] by its position p = positions[t]:
 *       window == 0  or  j > p - window  or  j < sinks
 *   new keys cached_lens[b] + j, j <= i, by bit j of its row of seen: any bits,
 *       not only those of attn_draft_tree
 *
 * Positions are cut to cached_lens[b] .. cached_lens[b] + i.  positions may not
 * be NULL; seen is [total_tokens, words], words 1 to 32.  max_new decides more
 * here: 33 to 256 rows of heads per key head have a kernel of their own, and
 * 0 counts all tokens as one sequence's.
 */
int attn_attend_tree(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks, int32_t max_blocks,
                     const void *q, int64_t q_stride, const void *k_cache, const void *v_cache,
                     const int32_t *table, const int32_t *cu_seqlens, const int32_t *cached_lens,
                     const int32_t *positions, const int32_t *seen, int32_t words,
                     float scale, int32_t window, int32_t sinks, int32_t max_new,
                     void *out, int64_t out_stride, float *lse,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The branch that the model agrees with: token 0 of a sequence, and from a kept
 * token on its first child whose token is the one chosen behind it.
 *
 *   tokens      [total_tokens]  int32 device: the drafted tokens
 *   parents     [total_tokens]  int32 device, as above
 *   choices     [total_tokens]  int32 device: the token that the model (or who
 *               samples from it) chose behind each
 *   path        [total_tokens]  int32 device, out: at cu_seqlens[b] + k the
 *               index of the k-th kept token, rising; -1 behind the last one
 *               and for tokens of no sequence
 *   counts      [batch]  int32 device, out: kept tokens, 0 without new ones
 *   next_tokens [batch]  int32 device, out: the token chosen behind the last
 *               kept one, which the next step begins with; -1 without new ones
 *   kept_lens   [batch]  int32 device, out: cached_lens[b] + counts[b]
 *
 * With a table (else NULL, and the last four are not read) the blocks that hold
 * only tokens that are not kept are given back, sequence by sequence and in the
 * order of a row's entries: free_blocks[n_free], and so on behind it; n_free_out
 * (one value, not n_free itself) is the new length, at most free_capacity.  Only
 * rows of a sequence's own blocks may be given back (attn_assign_blocks with
 * shared_tail sees to that).  The table stays as it is; nothing reads its
 * entries behind the cached tokens before they are handed out again.  Without
 * sequences nothing is written.
 */
int attn_accept_path(int32_t batch, int32_t block_size, int32_t max_blocks, int64_t total_tokens,
                     const int32_t *tokens, const int32_t *parents, const int32_t *choices,
                     const int32_t *cu_seqlens, const int32_t *cached_lens,
                     int32_t *path, int32_t *counts, int32_t *next_tokens, int32_t *kept_lens,
                     const int32_t *table, int32_t *free_blocks, int32_t free_capacity,
                     const int32_t *n_free, int32_t *n_free_out, void *hip_stream);

/*
 * The kept tokens' keys and values: in each of n_caches caches (the k_cache and
 * v_cache of every layer; a host array of device pointers, all of `shape`, none
 * of which overlap) row cached_lens[b] + path[k] is copied to row
 * cached_lens[b] + k, for k in rising order up to the first path[k] that is not
 * one of k .. n_b - 1.  Rows without a block are left out.  cached_lens are
 * those of the step, not kept_lens.  head_dim: as attn_rope_append; at most 256
 * caches.
 */
int attn_keep_path(const attn_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t n_blocks, int32_t max_blocks,
                   int32_t n_caches, void *const *caches, const int32_t *table,
                   const int32_t *cu_seqlens, const int32_t *cached_lens, const int32_t *path, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ATTN_TREE_H */
