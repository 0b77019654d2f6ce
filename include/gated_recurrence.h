/*
 * gated_recurrence.h -- C ABI of gated recurrent layers, the other kind of
 * recurrent layer that hybrid models put between their attention layers, on
 * MI355X (gfx950).
 *
 * Every channel is a recurrence of its own whose state keeps a part of itself
 * that two gates and a learned decay choose for every token:
 *
 *     a_t = exp(-sharpness softplus(decay) sigmoid(r_t))
 *     h_t = a_t h_(t-1) + sqrt(1 - a_t^2) sigmoid(i_t) x_t,     y_t = h_t
 *
 * What a prefix-cache hit resumes from is h, one row of fp32 per sequence
 * (Section 4.1: a recurrent layer is resumed from a whole state; Section 4.2:
 * states at chosen tokens become entries of the cache).  Operators:
 *
 *   rec_scan         packed sequences from initial states, states at chosen tokens
 *   rec_scan_grads   its backward pass
 *   rec_step         one token of every sequence, the states in place
 *   rec_step_tree    trees of drafted tokens (attn_tree.h), each token from its
 *                    parent's state
 *   rec_keep_states  the state behind the last token that was kept
 *
 * Gates, products and states are fp32; y and the gradients are rounded to the
 * type once.  Sigmoids and 1 - a^2 below 2^-126 count as 0.  A state that is not
 * finite stays so to the end of its sequence and reaches no other one.
 *
 * Sequence b of a packed batch is tokens cu_seqlens[b] .. cu_seqlens[b+1] - 1.
 * cu_seqlens [batch+1], int32 on the device, rises from 0 or more to at most
 * total_tokens; tokens outside belong to no sequence.  Lengths are read on the
 * device and nothing here allocates, copies to the host or synchronises, so
 * calls can be captured into a graph and replayed while the lengths change.  No
 * value of the device's index arrays makes a kernel access memory outside its
 * arguments.  A call takes at most 4096 sequences and 2^30 - 1 tokens, of which
 * rec_scan and rec_scan_grads have fewer than 2^23 blocks of 64 channels by 128
 * (rec_scan_grads: 64) tokens, of 128 channels where rows lie pair by pair.
 *
 * "device" pointers are HIP device pointers on the current device.  x, r, i, y
 * and dy are [total_tokens, channels] of io_dtype with `..._stride` elements
 * between tokens (at least channels, at most 2^22; for instance parts of the rows
 * of one projection), aligned to their type.  Every entry point returns REC_OK (0) or
 * a negative rec_status_t; on error nothing has been enqueued and
 * rec_last_error() returns a message for the calling thread.  Nothing here
 * throws or aborts.
 */
#ifndef GATED_RECURRENCE_H
#define GATED_RECURRENCE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    REC_OK = 0,
    REC_ERR_INVALID_ARG = -1,       /* NULL where a pointer is required, bad sizes */
    REC_ERR_UNSUPPORTED_SHAPE = -4, /* sizes outside what the kernels handle       */
    REC_ERR_WORKSPACE_TOO_SMALL = -5,
    REC_ERR_MISALIGNED = -6,
    REC_ERR_HIP = -7                /* a HIP runtime call failed                   */
} rec_status_t;

typedef enum { REC_DT_F32 = 0, REC_DT_BF16 = 1, REC_DT_F16 = 2 } rec_dtype_t;

typedef struct {
    int32_t channels; /* 1 to 2^20 */
    int32_t io_dtype; /* rec_dtype_t of x, r, i, y and their gradients */
    float sharpness;  /* positive and finite */
} rec_shape_t;

/* rows of `saved`: the states in front of every REC_SAVED_EVERY-th token */
#define REC_SAVED_EVERY 8

/*
 * Bytes of device workspace for rec_scan (grads = 0) or rec_scan_grads (grads
 * = 1, and 2 where it gets no `saved`) of a batch of this size.  The caller
 * allocates it, 256-byte aligned; its contents mean nothing between calls, and
 * calls that may run at the same time need workspaces of their own.
 */
int rec_workspace_bytes(const rec_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t grads, size_t *bytes);

/*
 *   decay         [channels]  fp32 device
 *   init_states   [batch, channels]  fp32 device, or NULL: zeros
 *   ckpt          [n_ckpt]  int32 device: packed tokens whose states are wanted,
 *                 in any order, more than once if need be; NULL if n_ckpt is 0.
 *                 Each is looked for among all: some hundreds per call cost
 *                 little, thousands many times the scan
 *   y             io_dtype, or NULL: not wanted.  Rows of tokens of no sequence
 *                 are not written.
 *   final_states  [batch, channels]  fp32 device, out, or NULL: behind a
 *                 sequence's last token; the initial state of one without tokens
 *   ckpt_states   [n_ckpt, channels]  fp32 device, out: the state behind token
 *                 ckpt[k]; zeros where that is a token of no sequence
 *   saved         [ceil(total_tokens / REC_SAVED_EVERY), channels]  fp32 device,
 *                 out, or NULL: what rec_scan_grads takes
 *
 * init_states may be final_states, and y may be x, r or i with its stride, as
 * in rec_step and rec_step_tree; apart from that nothing that is written
 * overlaps anything else.  Results do not depend on the timing of the GPU.
 */
int rec_scan(const rec_shape_t *shape, int32_t batch, int64_t total_tokens,
             const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i, int64_t i_stride,
             const float *decay, const int32_t *cu_seqlens, const float *init_states,
             const int32_t *ckpt, int32_t n_ckpt,
             void *y, int64_t y_stride, float *final_states, float *ckpt_states, float *saved,
             void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The gradients of a loss with respect to x, r, i, decay and the initial
 * states, from those with respect to y and the final states.
 *
 *   saved      what rec_scan wrote for the same inputs, or NULL: computed again
 *   dy         io_dtype, or NULL: zeros
 *   d_final    [batch, channels]  fp32 device, or NULL: zeros
 *   dx, dr, di [total_tokens, channels]  io_dtype, contiguous, out; zeros for
 *              tokens of no sequence
 *   d_decay    [channels]  fp32 device, out
 *   d_init     [batch, channels]  fp32 device, out, or NULL
 *
 * Where a gate or a decay leaves 1 - a^2 below 2^-126, the smallest normal fp32
 * value (sharpness softplus(decay) sigmoid(r) below 2^-127), it is taken as 0, and
 * so are the gradients through it, whose limit is 0.  Sums do not depend on the
 * timing of the GPU.
 */
int rec_scan_grads(const rec_shape_t *shape, int32_t batch, int64_t total_tokens,
                   const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i, int64_t i_stride,
                   const float *decay, const int32_t *cu_seqlens, const float *init_states, const float *saved,
                   const void *dy, int64_t dy_stride, const float *d_final,
                   void *dx, void *dr, void *di, float *d_decay, float *d_init,
                   void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * One token of every sequence: row b of x, r and i with row b of states
 * [batch, channels], fp32 device, which is replaced by the new state.
 */
int rec_step(const rec_shape_t *shape, int32_t batch,
             const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i, int64_t i_stride,
             const float *decay, float *states, void *y, int64_t y_stride, void *hip_stream);

/*
 * Trees of new tokens.  parents [total_tokens], int32 device: the index in its
 * sequence of the token whose state each continues, less than its own; -1, as
 * any other value: the sequence's row of states [batch, channels], which stays.
 *
 *   node_states [total_tokens, channels]  fp32 device, out: every token's state;
 *               like y's, rows of tokens of no sequence are not written
 */
int rec_step_tree(const rec_shape_t *shape, int32_t batch, int64_t total_tokens,
                  const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i, int64_t i_stride,
                  const float *decay, const float *states, const int32_t *cu_seqlens, const int32_t *parents,
                  void *y, int64_t y_stride, float *node_states, void *hip_stream);

/*
 * states[b] = node_states[cu_seqlens[b] + path[cu_seqlens[b] + counts[b] - 1]],
 * with path and counts as attn_accept_path writes them; a sequence without kept
 * tokens keeps its state.
 */
int rec_keep_states(int32_t channels, int32_t batch, int64_t total_tokens, float *states, const float *node_states,
                    const int32_t *cu_seqlens, const int32_t *path, const int32_t *counts, void *hip_stream);

/* Message of the last error on the calling thread ("" if none). */
const char *rec_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* GATED_RECURRENCE_H */
