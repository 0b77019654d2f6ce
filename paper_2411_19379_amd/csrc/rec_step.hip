// The gated recurrence of a few tokens: one of every sequence, the nodes of drafted trees, the state that is kept.
#include "rec_common.h"

namespace {

bool pairs(const void *p, int64_t stride, int bytes) { return reinterpret_cast<uintptr_t>(p) % (2 * bytes) == 0 && stride % 2 == 0; }

// ---------------------------------------------------------------- one token of every sequence
// V channels of a sequence per thread.  All latency up to some hundred sequences.
constexpr int kStepThreads = 128;
template <typename E, int V> __global__ __launch_bounds__(kStepThreads) void rec_step_kernel(RecIo in, const float *decay, float sharpness, int channels, float *states, void *y,
                                                                                            int64_t y_stride)
{
    const int c = (blockIdx.x * kStepThreads + threadIdx.x) * V;
    const int64_t b = blockIdx.y;
    if (c >= channels)
        return;
    typedef RecRow<E, V> Row;
    float x[V], r[V], i[V], h[V], d[V];
    Row::unpack(row_load<E, V>(in.x, b, in.x_stride, c), x);
    Row::unpack(row_load<E, V>(in.r, b, in.r_stride, c), r);
    Row::unpack(row_load<E, V>(in.i, b, in.i_stride, c), i);
    state_row_load<V>(states, b, channels, c, h);
    state_row_load<V>(decay, 0, channels, c, d);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const Gates g = gates_of(r[v], i[v], decay_rate(d[v], sharpness));
        h[v] = __builtin_fmaf(g.a, h[v], added(g, x[v])), pin(h[v]);
    }
    state_row_store<V>(states, b, channels, c, h);
    row_store<E, V>(y, b, y_stride, c, h);
}

// ---------------------------------------------------------------- trees
// A wave per sequence and 64 channels, kTreeAhead tokens at a time, whose inputs are requested while those in front are worked on.  Their
// gates, which are nearly all of the work and do not depend on states, are computed side by side; then the states, a product and
// a sum each, those of the last kNodes tokens kept in LDS for their children (older ones are read back).  Memory latency bounds it:
// 32 trees of 16 to 64 tokens of 4096 channels in bf16 23.5 us, of which the stores 6 and the gates 2 (two channels per thread and one
// token at a time 26.8, four waves that share a batch's gates 34); one tree of 17 tokens 6.9 us (8.6 and 6.0).
constexpr int kNodes = 64;
constexpr int kTreeAhead = 8;
template <typename E> __global__ __launch_bounds__(64) void rec_step_tree_kernel(RecIo in, const float *decay, float sharpness, int channels, const float *states, const int32_t *cu,
                                                                                const int32_t *parents, int64_t T, void *y, int64_t y_stride, float *node_states, int nodes)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    float *const lds = reinterpret_cast<float *>(lds_raw);  // [nodes][64]
    const int l = threadIdx.x, b = blockIdx.y;
    const RecSeq s = rec_seq(cu, b, T);
    const int own = blockIdx.x * 64 + l;
    const bool c_ok = own < channels;
    const int c = c_ok ? own : 0;
    if (s.n == 0)
        return;
    typedef RecRow<E, 1> Row;
    typename Row::Raw x[kTreeAhead], r[kTreeAhead], i[kTreeAhead];
    int parent = 0;  // of token l of the present and the next ones
    auto request = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kTreeAhead; ++u) {
            const int64_t t = s.start + (int64_t)(k0 + u < s.n ? k0 + u : s.n - 1);
            x[u] = row_load<E, 1>(in.x, t, in.x_stride, c);
            r[u] = row_load<E, 1>(in.r, t, in.r_stride, c);
            i[u] = row_load<E, 1>(in.i, t, in.i_stride, c);
        }
        if (k0 % 64 == 0)
            parent = parents[s.start + (int64_t)(k0 + l < s.n ? k0 + l : s.n - 1)];
    };
    const float rate = decay_rate(decay[c], sharpness), root = states[(int64_t)b * channels + c];
    float h = 0.f;
    request(0);
    for (int k0 = 0; k0 < s.n; k0 += kTreeAhead) {
        float kept[kTreeAhead], add[kTreeAhead];
        int from[kTreeAhead];
#pragma unroll
        for (int u = 0; u < kTreeAhead; ++u) {
            float xv, rv, iv;
            Row::unpack(x[u], &xv);
            Row::unpack(r[u], &rv);
            Row::unpack(i[u], &iv);
            const Gates g = gates_of(rv, iv, rate);
            kept[u] = g.a, add[u] = added(g, xv);
            from[u] = __builtin_amdgcn_readlane(parent, (k0 + u) % 64);
        }
        if (k0 + kTreeAhead < s.n)
            request(k0 + kTreeAhead);
#pragma unroll
        for (int u = 0; u < kTreeAhead; ++u) {
            const int k = k0 + u, p = from[u];
            if (k >= s.n)
                break;
            if (p != k - 1 || k == 0) {
                h = root;
                if (p >= 0 && p < k) {
                    if (k - p <= nodes) {
                        h = lds[p % nodes * 64 + l];
                    } else {
                        h = node_states[(s.start + (int64_t)p) * channels + c];
                        pin(h);  // waited for here: behind the branch every token would wait for all loads and stores on their way
                    }
                }
            }
            h = __builtin_fmaf(kept[u], h, add[u]), pin(h);
            lds[k % nodes * 64 + l] = h;
            if (c_ok) {
                row_store<E, 1>(y, s.start + (int64_t)k, y_stride, own, &h);
                node_states[(s.start + (int64_t)k) * channels + own] = h;
            }
        }
    }
}

// ---------------------------------------------------------------- the state behind the last kept token
constexpr int kKeepThreads = 256;
__global__ __launch_bounds__(kKeepThreads) void rec_keep_kernel(int channels, int64_t T, float *states, const float *node_states, const int32_t *cu, const int32_t *path,
                                                               const int32_t *counts)
{
    const int b = blockIdx.y, c = blockIdx.x * kKeepThreads + threadIdx.x;
    const RecSeq s = rec_seq(cu, b, T);
    const int count = counts[b];
    if (c >= channels || count < 1 || count > s.n)
        return;
    const int last = path[s.start + (int64_t)count - 1];
    if (last >= 0 && last < s.n)
        states[(int64_t)b * channels + c] = node_states[(s.start + (int64_t)last) * channels + c];
}

template <typename E, int V> hipError_t step(const rec_shape_t &s, int batch, const RecIo &in, const float *decay, float *states, void *y, int64_t y_stride, hipStream_t stream)
{
    const int per = kStepThreads * V;
    hipLaunchKernelGGL((rec_step_kernel<E, V>), dim3((unsigned)((s.channels + per - 1) / per), (unsigned)batch), dim3(kStepThreads), 0, stream, in, decay, s.sharpness,
                       s.channels, states, y, y_stride);
    return hipGetLastError();
}
template <typename E> hipError_t step_tree(const rec_shape_t &s, int batch, int64_t T, const RecIo &in, const float *decay, const float *states, const int32_t *cu,
                                           const int32_t *parents, void *y, int64_t y_stride, float *node_states, hipStream_t stream)
{
    const int nodes = T < kNodes ? (int)T : kNodes;
    hipLaunchKernelGGL((rec_step_tree_kernel<E>), dim3((unsigned)((s.channels + 63) / 64), (unsigned)batch), dim3(64), (size_t)nodes * 64 * sizeof(float), stream, in, decay,
                       s.sharpness, s.channels, states, cu, parents, T, y, y_stride, node_states, nodes);
    return hipGetLastError();
}

bool two_channels(const rec_shape_t &s, const RecIo &in, const void *y, int64_t y_stride, const float *decay, const float *states)
{
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    return s.channels % 2 == 0 && pairs(in.x, in.x_stride, e) && pairs(in.r, in.r_stride, e) && pairs(in.i, in.i_stride, e) && pairs(y, y_stride, e) && pairs(decay, 0, 4) &&
           pairs(states, 0, 4);
}

}  // namespace

hipError_t launch_rec_step(const rec_shape_t &s, int batch, const RecIo &in, const float *decay, float *states, void *y, int64_t y_stride, hipStream_t stream)
{
    const bool two = two_channels(s, in, y, y_stride, decay, states);
    if (s.io_dtype == REC_DT_F32)
        return two ? step<RecF32, 2>(s, batch, in, decay, states, y, y_stride, stream) : step<RecF32, 1>(s, batch, in, decay, states, y, y_stride, stream);
    if (s.io_dtype == REC_DT_BF16)
        return two ? step<RecBf16, 2>(s, batch, in, decay, states, y, y_stride, stream) : step<RecBf16, 1>(s, batch, in, decay, states, y, y_stride, stream);
    return two ? step<RecF16, 2>(s, batch, in, decay, states, y, y_stride, stream) : step<RecF16, 1>(s, batch, in, decay, states, y, y_stride, stream);
}

hipError_t launch_rec_step_tree(const rec_shape_t &s, int batch, int64_t T, const RecIo &in, const float *decay, const float *states, const int32_t *cu,
                                const int32_t *parents, void *y, int64_t y_stride, float *node_states, hipStream_t stream)
{
    if (s.io_dtype == REC_DT_F32)
        return step_tree<RecF32>(s, batch, T, in, decay, states, cu, parents, y, y_stride, node_states, stream);
    if (s.io_dtype == REC_DT_BF16)
        return step_tree<RecBf16>(s, batch, T, in, decay, states, cu, parents, y, y_stride, node_states, stream);
    return step_tree<RecF16>(s, batch, T, in, decay, states, cu, parents, y, y_stride, node_states, stream);
}

hipError_t launch_rec_keep(int channels, int batch, int64_t T, float *states, const float *node_states, const int32_t *cu, const int32_t *path, const int32_t *counts,
                           hipStream_t stream)
{
    hipLaunchKernelGGL(rec_keep_kernel, dim3((unsigned)((channels + kKeepThreads - 1) / kKeepThreads), (unsigned)batch), dim3(kKeepThreads), 0, stream, channels, T, states,
                       node_states, cu, path, counts);
    return hipGetLastError();
}
