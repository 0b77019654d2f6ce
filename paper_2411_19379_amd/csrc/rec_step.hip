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
// a sum each, those of the last kNodes tokens kept in LDS for their children (older ones are read back).  The longest tree bounds it,
// a batch of tokens 2 us, half of them gates on the vector units: 32 trees of 16 to 64 tokens of 4096 channels in bf16 19.8 us, 8 of
// 256 tokens 62, one of 17 tokens 6.2 (stores and requests in branches, so that inputs are waited for together with all stores, 23.6,
// 85 and 6.9; two channels per thread and one token at a time 26.8, 103 and 8.6; four waves that share a batch's gates 34, 78 and 6.0;
// inputs requested two batches ahead no faster; 16 tokens at a time 20.8, 60 and 7.4).
constexpr int kNodes = 64;
constexpr int kTreeAhead = 8;
template <typename E> __global__ __launch_bounds__(64) void rec_step_tree_kernel(RecIo in, const float *decay, float sharpness, int channels, const float *states, const int32_t *cu,
                                                                                const int32_t *parents, int64_t T, void *y, int64_t y_stride, float *node_states)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    float *const lds = reinterpret_cast<float *>(lds_raw);  // [kNodes][64]
    const int l = threadIdx.x, b = blockIdx.y;
    const RecSeq s = rec_seq(cu, b, T);
    const int own = blockIdx.x * 64 + l, c = own < channels ? own : channels - 1;  // lanes without a channel do the last one's work once more
    if (s.n == 0)
        return;
    typedef RecRow<E, 1> Row;
    typename Row::Raw x[kTreeAhead], r[kTreeAhead], i[kTreeAhead];
    int parent = 0;  // of token l of the next ones
    auto request = [&](int from) __attribute__((always_inline)) {  // tokens behind the last one are read from that
        const int k0 = from < s.n ? from : s.n - 1, rows = s.n - k0 < kTreeAhead ? s.n - k0 : kTreeAhead;
        const int64_t t = s.start + (int64_t)k0;
        const WaveRows<E> x_rows(in.x, t, in.x_stride, rows, channels), r_rows(in.r, t, in.r_stride, rows, channels), i_rows(in.i, t, in.i_stride, rows, channels);
        const uint32_t at = x_rows.at(0, c);
#pragma unroll
        for (int u = 0; u < kTreeAhead; ++u) {
            const int row = u < rows ? u : rows - 1;
            x_rows.get(at, row, x[u]);
            r_rows.get(at, row, r[u]);
            i_rows.get(at, row, i[u]);
        }
        parent = parents[t + (l < rows ? l : rows - 1)];
    };
    const float rate = decay_rate(decay[c], sharpness), root = states[(int64_t)b * channels + c];
    float h = 0.f;
    request(0);
    for (int k0 = 0; k0 < s.n; k0 += kTreeAhead) {
        const int rows = s.n - k0 < kTreeAhead ? s.n - k0 : kTreeAhead;
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
            from[u] = __builtin_amdgcn_readlane(parent, u);
        }
        request(k0 + kTreeAhead);
        const int64_t t = s.start + (int64_t)k0;
        const WaveRows<E> y_rows(y, t, y_stride, rows, channels);
        const WaveRows<RecF32> node_rows(node_states, t, channels, rows, channels);
        const uint32_t y_at = y_rows.at(0, c), node_at = node_rows.at(0, c);
#pragma unroll
        for (int u = 0; u < kTreeAhead; ++u) {
            const int k = k0 + u, p = u < rows ? from[u] : k - 1, row = u < rows ? u : rows - 1;
            if (p != k - 1 || k == 0) {
                h = root;
                if (p >= 0 && p < k) {
                    if (k - p <= kNodes) {
                        h = lds[(p & (kNodes - 1)) * 64 + l];
                    } else {
                        h = node_states[(s.start + (int64_t)p) * channels + c];
                        pin(h);  // waited for here: behind the branch every token would wait for all loads and stores on their way
                    }
                }
            }
            const float next = __builtin_fmaf(kept[u], h, add[u]);
            h = u < rows ? next : h, pin(h);
            lds[(k & (kNodes - 1)) * 64 + l] = h;
            // No branch around the stores (behind the last token its own are repeated), nor around the requests: what waits for inputs
            // would wait for everything behind them if their number were not known.
            y_rows.put(y_at, row, Row::pack(&h));
            node_rows.put(node_at, row, __float_as_uint(h));
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
    hipLaunchKernelGGL((rec_step_tree_kernel<E>), dim3((unsigned)((s.channels + 63) / 64), (unsigned)batch), dim3(64), kNodes * 64 * sizeof(float), stream, in, decay,
                       s.sharpness, s.channels, states, cu, parents, T, y, y_stride, node_states);
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
