// What the kernels of the gated recurrence share (gfx950 only): gates, rows of channels in their types, sequences.
#pragma once

#include "gated_recurrence.h"
#include "mfma_utils.h"

// Products and sums are put together where it is written, and nowhere else: code that is compiled twice, with and without the ends of
// sequences in it, rounds alike.
#pragma clang fp contract(off)

namespace {

constexpr int kRecMaxBatch = 4096;

// LDS is ordered, loads in flight stay in flight
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The value is in a register from here on.  What is computed from it behind is not computed in front (the compiler would do so for
// all tokens of a wave and have no registers for it), and it has been rounded to fp32 (a product and sum that go to fp16 would be
// rounded once there, and differently where the same code is compiled with something between the two).
__device__ __forceinline__ void pin(float &v) { asm volatile("" : "+v"(v)); }

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
    typedef uint32_t Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = __uint_as_float(r); }
    static __device__ __forceinline__ Raw pack(const float *v) { return __float_as_uint(v[0]); }
};
template <> struct RecRow<RecF32, 2> {
    typedef uint2 Raw;
    static __device__ __forceinline__ void unpack(Raw r, float *v) { v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y); }
    static __device__ __forceinline__ Raw pack(const float *v) { return make_uint2(__float_as_uint(v[0]), __float_as_uint(v[1])); }
};
// Channels c .. c + V - 1 of row t.
template <typename E, int V> __device__ __forceinline__ typename RecRow<E, V>::Raw row_load(const void *base, int64_t t, int64_t stride, int c)
{
    return *reinterpret_cast<const typename RecRow<E, V>::Raw *>(static_cast<const unsigned char *>(base) + (t * stride + c) * E::kBytes);
}
template <typename E, int V> __device__ __forceinline__ void row_store(void *base, int64_t t, int64_t stride, int c, const float *v)
{
    *reinterpret_cast<typename RecRow<E, V>::Raw *>(static_cast<unsigned char *>(base) + (t * stride + c) * E::kBytes) = RecRow<E, V>::pack(v);
}
// The same for a wave's rows, through a descriptor: a row is a uniform offset and a lane's place in it one that does not change, so
// that no address is computed on the vector ALUs (with pointers these were a quarter of the instructions of a token).  A wave's
// rows span less than 2^31 bytes, since strides are at most kRecMostStride.
constexpr int64_t kRecMostStride = 1 << 22;
template <typename E> struct WaveRows {
    rsrc_t rows;
    uint32_t stride;  // bytes
    // `n` rows from row t on, of `channels` channels
    __device__ __forceinline__ WaveRows(const void *base, int64_t t, int64_t stride_, int n, int channels)
        : rows(make_rsrc(static_cast<const unsigned char *>(base) + t * stride_ * E::kBytes, ((uint32_t)(n - 1) * (uint32_t)stride_ + (uint32_t)channels) * E::kBytes)),
          stride((uint32_t)stride_ * E::kBytes)
    {
    }
    // a lane's offset: channel c of row `row`
    __device__ __forceinline__ uint32_t at(int row, int c) const { return (uint32_t)row * stride + (uint32_t)c * E::kBytes; }
    __device__ __forceinline__ void get(uint32_t at, int row, uint16_t &r) const { r = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rows, (int)at, (int)(row * stride), 0); }
    __device__ __forceinline__ void get(uint32_t at, int row, uint32_t &r) const { r = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rows, (int)at, (int)(row * stride), 0); }
    __device__ __forceinline__ void get(uint32_t at, int row, uint2 &r) const
    {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(rows, (int)at, (int)(row * stride), 0);
        r = make_uint2(v[0], v[1]);
    }
    __device__ __forceinline__ void put(uint32_t at, int row, uint16_t r) const { __builtin_amdgcn_raw_buffer_store_b16(r, rows, (int)at, (int)(row * stride), 0); }
    __device__ __forceinline__ void put(uint32_t at, int row, uint32_t r) const { __builtin_amdgcn_raw_buffer_store_b32(r, rows, (int)at, (int)(row * stride), 0); }
    __device__ __forceinline__ void put(uint32_t at, int row, uint2 r) const
    {
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 v = {r.x, r.y};
        __builtin_amdgcn_raw_buffer_store_b64(v, rows, (int)at, (int)(row * stride), 0);
    }
};
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
// 1 - a^2 = -expm1(2 log a), whose value counts where a is next to 1: up to v = -2 log a = 1/4 as v times the polynomial of degree 4
// that is next to (1 - e^-v) / v there (3e-9 of it, found by exchanging extrema), and 1 - a a, which loses two bits at most, behind.
// (1 - a from a in fp32 has lost all of them at a = 1 - 2^-24.)
__device__ __forceinline__ float one_minus_square(float log2_a, float a)
{
    const float v = log2_a * -1.38629436111989062f;
    float near = __builtin_fmaf(v, 0.007510221719597369f, -0.041488954085247894f);
    near = __builtin_fmaf(v, near, 0.16665081472713647f);
    near = __builtin_fmaf(v, near, -0.49999950132422216f);
    near = v * __builtin_fmaf(v, near, 1.f);
    return v < 0.25f ? near : __builtin_fmaf(-a, a, 1.f);
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
// Whether a launch can number the workgroups of T tokens, where rows allow the most channels in each, and of these rows.
bool rec_fits(const rec_shape_t &s, int64_t T, int grads);
bool rec_fits(const rec_shape_t &s, const RecScan &a);
bool rec_fits(const rec_shape_t &s, const RecGrads &a);
hipError_t launch_rec_scan(const rec_shape_t &s, const RecScan &a, void *workspace, hipStream_t stream);
hipError_t launch_rec_grads(const rec_shape_t &s, const RecGrads &a, void *workspace, hipStream_t stream);
hipError_t launch_rec_step(const rec_shape_t &s, int batch, const RecIo &in, const float *decay, float *states, void *y, int64_t y_stride,
                           hipStream_t stream);
hipError_t launch_rec_step_tree(const rec_shape_t &s, int batch, int64_t T, const RecIo &in, const float *decay, const float *states,
                                const int32_t *cu, const int32_t *parents, void *y, int64_t y_stride, float *node_states,
                                hipStream_t stream);
hipError_t launch_rec_keep(int channels, int batch, int64_t T, float *states, const float *node_states, const int32_t *cu,
                           const int32_t *path, const int32_t *counts, hipStream_t stream);
