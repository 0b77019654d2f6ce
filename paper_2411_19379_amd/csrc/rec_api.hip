// Entry points of the gated recurrence: argument checks and launches.  Nothing here allocates or synchronises.
#include <cmath>
#include <initializer_list>
#include <string>

#include "rec_common.h"

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

int hip_status(hipError_t e) { return e == hipSuccess ? (int)REC_OK : fail(REC_ERR_HIP, hipGetErrorString(e)); }

int check_shape(const rec_shape_t *s)
{
    if (!s)
        return fail(REC_ERR_INVALID_ARG, "shape is NULL");
    if (s->channels < 1)
        return fail(REC_ERR_INVALID_ARG, "channels must be positive");
    if (s->channels > 1 << 20)
        return fail(REC_ERR_UNSUPPORTED_SHAPE, "at most 2^20 channels");
    if (s->io_dtype != REC_DT_F32 && s->io_dtype != REC_DT_BF16 && s->io_dtype != REC_DT_F16)
        return fail(REC_ERR_INVALID_ARG, "io_dtype is not one of rec_dtype_t");
    if (!(s->sharpness > 0.f) || !std::isfinite(s->sharpness))
        return fail(REC_ERR_INVALID_ARG, "sharpness must be positive and finite");
    return REC_OK;
}

int check_batch(int32_t batch, int64_t total_tokens)
{
    if (batch < 0 || total_tokens < 0)
        return fail(REC_ERR_INVALID_ARG, "batch and total_tokens must not be negative");
    if (batch > kRecMaxBatch)
        return fail(REC_ERR_UNSUPPORTED_SHAPE, "at most 4096 sequences per call");
    if (total_tokens > 0x3fffffff)
        return fail(REC_ERR_UNSUPPORTED_SHAPE, "at most 2^30 - 1 tokens per call");
    if (batch == 0 && total_tokens > 0)
        return fail(REC_ERR_INVALID_ARG, "tokens without sequences");
    return REC_OK;
}

int check_fits(bool fits)
{
    return fits ? (int)REC_OK : fail(REC_ERR_UNSUPPORTED_SHAPE, "tokens and channels take more workgroups than a launch has: 2^23 - 1 of 64 channels and 128 tokens, 64 for gradients");
}

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Rows of channels every `stride` elements.
int check_rows(const rec_shape_t &s, const void *p, int64_t stride, const char *what)
{
    if (!p)
        return fail(REC_ERR_INVALID_ARG, what);
    if (stride < s.channels || stride > kRecMostStride)
        return fail(REC_ERR_INVALID_ARG, "a token stride is shorter than the channels, or beyond 2^22");
    if (!aligned(p, s.io_dtype == REC_DT_F32 ? 4 : 2))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    return REC_OK;
}

int check_inputs(const rec_shape_t &s, const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i, int64_t i_stride)
{
    int rc = check_rows(s, x, x_stride, "x is NULL");
    if (rc == REC_OK)
        rc = check_rows(s, r, r_stride, "r is NULL");
    if (rc == REC_OK)
        rc = check_rows(s, i, i_stride, "i is NULL");
    return rc;
}

bool floats(std::initializer_list<const void *> all)
{
    for (const void *p : all)
        if (!aligned(p, 4))
            return false;
    return true;
}

int check_workspace(const rec_shape_t &s, int32_t batch, int64_t total_tokens, int grads, const void *workspace, size_t bytes)
{
    const size_t need = rec_scan_workspace(s, batch, total_tokens, grads);
    if (need && (!workspace || bytes < need))
        return fail(REC_ERR_WORKSPACE_TOO_SMALL, "workspace is NULL or smaller than rec_workspace_bytes");
    if (need && !aligned(workspace, 256))
        return fail(REC_ERR_MISALIGNED, "workspace is not 256-byte aligned");
    return REC_OK;
}

}  // namespace

extern "C" const char *rec_last_error(void) { return g_error.c_str(); }

extern "C" int rec_workspace_bytes(const rec_shape_t *shape, int32_t batch, int64_t total_tokens, int32_t grads, size_t *bytes)
{
    int rc = check_shape(shape);
    if (rc == REC_OK)
        rc = check_batch(batch, total_tokens);
    if (rc != REC_OK)
        return rc;
    if (!bytes || grads < 0 || grads > 2)
        return fail(REC_ERR_INVALID_ARG, "bytes is NULL or grads not one of 0, 1, 2");
    rc = check_fits(rec_fits(*shape, total_tokens, grads));
    if (rc != REC_OK)
        return rc;
    *bytes = rec_scan_workspace(*shape, batch, total_tokens, grads);
    return REC_OK;
}

extern "C" int rec_scan(const rec_shape_t *shape, int32_t batch, int64_t total_tokens, const void *x, int64_t x_stride, const void *r, int64_t r_stride,
                        const void *i, int64_t i_stride, const float *decay, const int32_t *cu_seqlens, const float *init_states,
                        const int32_t *ckpt, int32_t n_ckpt, void *y, int64_t y_stride, float *final_states, float *ckpt_states,
                        float *saved, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == REC_OK)
        rc = check_batch(batch, total_tokens);
    if (rc != REC_OK)
        return rc;
    if (n_ckpt < 0 || (n_ckpt > 0 && (!ckpt || !ckpt_states)))
        return fail(REC_ERR_INVALID_ARG, "ckpt and ckpt_states are required where n_ckpt is positive");
    if (!floats({decay, init_states, final_states, ckpt_states, saved}))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    if (batch == 0)
        return n_ckpt == 0 ? (int)REC_OK : fail(REC_ERR_INVALID_ARG, "checkpoints without sequences");
    RecScan a;
    a.in = RecIo{x, r, i, x_stride, r_stride, i_stride};
    a.decay = decay, a.init = init_states, a.cu = cu_seqlens, a.ckpt = ckpt;
    a.y = y, a.y_stride = y_stride, a.final_states = final_states, a.ckpt_states = ckpt_states, a.saved = saved;
    a.T = total_tokens, a.batch = batch, a.n_ckpt = n_ckpt;
    if (total_tokens > 0) {
        rc = check_inputs(*shape, x, x_stride, r, r_stride, i, i_stride);
        if (rc == REC_OK && y)
            rc = check_rows(*shape, y, y_stride, "y is NULL");
        if (rc == REC_OK && (!decay || !cu_seqlens))
            rc = fail(REC_ERR_INVALID_ARG, "decay or cu_seqlens is NULL");
        if (rc == REC_OK)
            rc = check_fits(rec_fits(*shape, a));
        if (rc == REC_OK)
            rc = check_workspace(*shape, batch, total_tokens, 0, workspace, workspace_bytes);
        if (rc != REC_OK)
            return rc;
    }
    return hip_status(launch_rec_scan(*shape, a, workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int rec_scan_grads(const rec_shape_t *shape, int32_t batch, int64_t total_tokens, const void *x, int64_t x_stride, const void *r,
                              int64_t r_stride, const void *i, int64_t i_stride, const float *decay, const int32_t *cu_seqlens,
                              const float *init_states, const float *saved, const void *dy, int64_t dy_stride, const float *d_final,
                              void *dx, void *dr, void *di, float *d_decay, float *d_init, void *workspace, size_t workspace_bytes,
                              void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == REC_OK)
        rc = check_batch(batch, total_tokens);
    if (rc != REC_OK)
        return rc;
    if (!decay || !d_decay)
        return fail(REC_ERR_INVALID_ARG, "decay or d_decay is NULL");
    if (!floats({decay, init_states, saved, d_final, d_decay, d_init}))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    RecGrads a;
    a.in = RecIo{x, r, i, x_stride, r_stride, i_stride};
    a.decay = decay, a.init = init_states, a.saved = saved, a.d_final = d_final, a.cu = cu_seqlens;
    a.dy = dy, a.dy_stride = dy_stride, a.dx = dx, a.dr = dr, a.di = di, a.d_decay = d_decay, a.d_init = d_init;
    a.T = total_tokens, a.batch = batch;
    if (total_tokens > 0) {
        rc = check_inputs(*shape, x, x_stride, r, r_stride, i, i_stride);
        if (rc == REC_OK && dy)
            rc = check_rows(*shape, dy, dy_stride, "dy is NULL");
        for (const void *to : {dx, dr, di})
            if (rc == REC_OK)
                rc = check_rows(*shape, to, shape->channels, "dx, dr or di is NULL");
        if (rc == REC_OK && !cu_seqlens)
            rc = fail(REC_ERR_INVALID_ARG, "cu_seqlens is NULL");
        if (rc == REC_OK)
            rc = check_fits(rec_fits(*shape, a));
        if (rc == REC_OK)
            rc = check_workspace(*shape, batch, total_tokens, saved ? 1 : 2, workspace, workspace_bytes);
        if (rc != REC_OK)
            return rc;
    }
    return hip_status(launch_rec_grads(*shape, a, workspace, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int rec_step(const rec_shape_t *shape, int32_t batch, const void *x, int64_t x_stride, const void *r, int64_t r_stride, const void *i,
                        int64_t i_stride, const float *decay, float *states, void *y, int64_t y_stride, void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == REC_OK)
        rc = check_batch(batch, 0);
    if (rc != REC_OK || batch == 0)
        return rc;
    rc = check_inputs(*shape, x, x_stride, r, r_stride, i, i_stride);
    if (rc == REC_OK)
        rc = check_rows(*shape, y, y_stride, "y is NULL");
    if (rc != REC_OK)
        return rc;
    if (!decay || !states)
        return fail(REC_ERR_INVALID_ARG, "decay or states is NULL");
    if (!floats({decay, states}))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    return hip_status(launch_rec_step(*shape, batch, RecIo{x, r, i, x_stride, r_stride, i_stride}, decay, states, y, y_stride,
                                      static_cast<hipStream_t>(hip_stream)));
}

extern "C" int rec_step_tree(const rec_shape_t *shape, int32_t batch, int64_t total_tokens, const void *x, int64_t x_stride, const void *r,
                             int64_t r_stride, const void *i, int64_t i_stride, const float *decay, const float *states,
                             const int32_t *cu_seqlens, const int32_t *parents, void *y, int64_t y_stride, float *node_states,
                             void *hip_stream)
{
    int rc = check_shape(shape);
    if (rc == REC_OK)
        rc = check_batch(batch, total_tokens);
    if (rc != REC_OK || total_tokens == 0)
        return rc;
    rc = check_inputs(*shape, x, x_stride, r, r_stride, i, i_stride);
    if (rc == REC_OK)
        rc = check_rows(*shape, y, y_stride, "y is NULL");
    if (rc != REC_OK)
        return rc;
    if (!decay || !states || !cu_seqlens || !parents || !node_states)
        return fail(REC_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!floats({decay, states, node_states}))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    return hip_status(launch_rec_step_tree(*shape, batch, total_tokens, RecIo{x, r, i, x_stride, r_stride, i_stride}, decay, states, cu_seqlens,
                                           parents, y, y_stride, node_states, static_cast<hipStream_t>(hip_stream)));
}

extern "C" int rec_keep_states(int32_t channels, int32_t batch, int64_t total_tokens, float *states, const float *node_states,
                               const int32_t *cu_seqlens, const int32_t *path, const int32_t *counts, void *hip_stream)
{
    const int rc = check_batch(batch, total_tokens);
    if (rc != REC_OK || total_tokens == 0)
        return rc;
    if (channels < 1 || channels > 1 << 20)
        return fail(REC_ERR_UNSUPPORTED_SHAPE, "1 to 2^20 channels");
    if (!states || !node_states || !cu_seqlens || !path || !counts)
        return fail(REC_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!floats({states, node_states}))
        return fail(REC_ERR_MISALIGNED, "a device pointer is not aligned to its type");
    return hip_status(launch_rec_keep(channels, batch, total_tokens, states, node_states, cu_seqlens, path, counts,
                                      static_cast<hipStream_t>(hip_stream)));
}
