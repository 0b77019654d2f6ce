// What the kernels of the gated recurrence share (gfx950 only): gates, rows of channels in their types, sequences.
#pragma once

#include "gated_recurrence.h"
#include "mfma_utils.h"

namespace {

constexpr int kRecMaxBatch = 4096;

// LDS is ordered, loads in flight stay in flight
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---------------------------------------------------------------- V neighbouring channels of a token
struct RecF32 {
    static constexpr int kBytes = 4;
};
struct RecBf16 {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float lo(uint32_t u) { return bf16_lo(u); }
    static __device__ __forceinline__ float hi(uint32_t u) { return bf16_hi(u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2_bf16(a, b); }
};
struct RecF16 {
    static constexpr int kBytes = 2;
    static __device__ __forceinline__ float lo(uint32_t u) { return f16_lo(u); }
    static __device__ __forceinline__ float hi(uint32_t u) { return f16_hi(u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack2_f16(a, b); }
};
template <typename E, int V> struct RecRow;
template <typename E> struct RecRow<E, 1> {
    typedef uint16_t Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = E::lo(r); }
    static __device__ __forceinline__ Raw pack(const float *v) { return (Raw)E::pack(v[0], 0.f); }
};
template <typename E> struct RecRow<E, 2> {
    typedef uint32_t Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = E::lo(r), v[1] = E::hi(r); }
    static __device__ __forceinline__ Raw pack(const float *v) { return E::pack(v[0], v[1]); }
};
template <> struct RecRow<RecF32, 1> {
    typedef float Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = r; }
    static __device__ __forceinline__ Raw pack(const float *v) { return v[0]; }
};
template <> struct RecRow<RecF32, 2> {
    typedef float2 Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = r.x, v[1] = r.y; }
    static __device__ __forceinline__ Raw pack(const float *v) { return make_float2(v[0], v[1]); }
};
// Channels c .. c + V - 1 of row t.
template <typename E, int V> __device__ __forceinline__ typename RecRow<E, V>::Raw row_load(const void *base, int64_t t, int64_t stride, int c)
{
    return *reinterpret_cast<const typename RecRow<E, V>::Raw *>(static_cast<const unsigned char *>(base) + t * stride * E::kBytes + (uint32_t)c * E::kBytes);
}
template <typename E, int V> __device__ __forceinline__ void row_store(void *base, int64_t t, int64_t stride, int c, const float *v)
{
    *reinterpret_cast<typename RecRow<E, V>::Raw *>(static_cast<unsigned char *>(base) + t * stride * E::kBytes + (uint32_t)c * E::kBytes) = RecRow<E, V>::pack(v);
}
template <int V> __device__ __forceinline__ void state_row_load(const float *base, int64_t row, int channels, int c, float *v)
{
    RecRow<RecF32, V>::unpack(row_load<RecF32, V>(base, row, channels, c), v);
}
template <int V> __device__ __forceinline__ void state_row_store(float *base, int64_t row, int channels, int c, const float *v)
{
    row_store<RecF32, V>(base, row, channels, c, v);
}

// ---------------------------------------------------------------- gates
// log2 of a per unit of sigmoid(r): -sharpness softplus(decay) log2(e)
__device__ __forceinline__ float decay_rate(float decay, float sharpness)
{
    return -sharpness * (fmaxf(decay, 0.f) + log1pf(expf(-fabsf(decay)))) * kLog2e;
}
__device__ __forceinline__ float sigmoid_fast(float v) { return __builtin_amdgcn_rcpf(1.f + exp2_fast(-kLog2e * v)); }
// 1 - a^2 = -expm1(2 log a), whose value counts where a is next to 1: a series to the sixth power up to 2 log a = -1/4, where the
// next term is 5e-8 of it; 1 - a a, which loses two bits at most, behind.  (a - 1 from a in fp32 has lost them all at a = 1 - 2^-24.)
__device__ __forceinline__ float one_minus_square(float log2_a, float a)
{
    const float v = log2_a * -1.38629436111989062f;  // -2 log a
    const float series = v * (1.f + v * (-1.f / 2 + v * (1.f / 6 + v * (-1.f / 24 + v * (1.f / 120 + v * (-1.f / 720))))));
    return v < 0.25f ? series : __builtin_fmaf(-a, a, 1.f);
}
struct Gates {
    float a;      // what the state keeps
    float log2_a;
    float sr, si; // sigmoids of the gates
    float kept2;  // 1 - a^2
};
__device__ __forceinline__ Gates gates_of(float r, float i, float rate)
{
    Gates g;
    g.sr = sigmoid_fast(r);
    g.si = sigmoid_fast(i);
    g.log2_a = rate * g.sr;
    g.a = exp2_fast(g.log2_a);
    g.kept2 = one_minus_square(g.log2_a, g.a);
    return g;
}
// What a token adds to the state.
__device__ __forceinline__ float added(const Gates &g, float x) { return __builtin_amdgcn_sqrtf(g.kept2) * g.si * x; }

// ---------------------------------------------------------------- sequences
struct RecSeq {
    int start, n;
};
__device__ __forceinline__ RecSeq rec_seq(const int32_t *cu, int b, int64_t T)
{
    const int from = cu[b] < 0 ? 0 : cu[b], to = cu[b + 1] > T ? (int)T : cu[b + 1];
    RecSeq s;
    s.start = from;
    s.n = to > from ? to - from : 0;
    return s;
}

}  // namespace

struct RecIo {
    const void *x, *r, *i;
    int64_t x_stride, r_stride, i_stride;
};
struct RecScan {
    RecIo in;
    const float *decay, *init;
    const int32_t *cu, *ckpt;
    void *y;
    int64_t y_stride;
    float *final_states, *ckpt_states, *saved;
    int64_t T;
    int32_t batch, n_ckpt;
};
struct RecGrads {
    RecIo in;
    const float *decay, *init, *saved, *d_final;
    const int32_t *cu;
    const void *dy;
    int64_t dy_stride;
    void *dx, *dr, *di;
    float *d_decay, *d_init;
    int64_t T;
    int32_t batch;
};
// Launchers implemented next to their kernels.
size_t rec_scan_workspace(const rec_shape_t &s, int batch, int64_t T, int grads);
hipError_t launch_rec_scan(const rec_shape_t &s, const RecScan &a, void *workspace, hipStream_t stream);
hipError_t launch_rec_grads(const rec_shape_t &s, const RecGrads &a, void *workspace, hipStream_t stream);
hipError_t launch_rec_step(const rec_shape_t &s, int batch, const RecIo &in, const float *decay, float *states, void *y, int64_t y_stride,
                           hipStream_t stream);
hipError_t launch_rec_step_tree(const rec_shape_t &s, int batch, int64_t T, const RecIo &in, const float *decay, const float *states,
                                const int32_t *cu, const int32_t *parents, void *y, int64_t y_stride, float *node_states,
                                hipStream_t stream);
hipError_t launch_rec_keep(int channels, int batch, int64_t T, float *states, const float *node_states, const int32_t *cu,
                           const int32_t *path, const int32_t *counts, hipStream_t stream);
