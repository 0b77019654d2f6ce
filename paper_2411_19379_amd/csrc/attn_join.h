// How the work of an attention launch is dealt out and its partial results are joined: what the kernels of attn_attend.hip and
// attn_tree_attend.hip share.  attn_common.h is included in front of it.
#pragma once

#include <cfloat>

#ifndef ATTN_TARGET  // workgroups that a launch is dealt to, where tests do not choose them
#define ATTN_TARGET 0
#endif

namespace {

constexpr float kOutgrown = 8.f;  // powers of two by which a weight may exceed that of the maximum before its row is scaled down

// ================================================================ joining
// The rows of sequences whose keys were split, a wave per row: the lanes load the maxima and weights of up to 64 parts at once,
// then the sums in the order of the parts, 64 * 4 / D parts per load and kJoinAhead loads on their way.  Two dependent trips to
// memory bound it (a chat turn's 4384 rows of 10 parts: 10 us; two rows per wave at once were 2 us faster there and 4 us slower
// for few rows of many parts).
constexpr int kJoinThreads = 256;
constexpr int kJoinAhead = 4;
constexpr int kJoinWorkgroups = 2048;

template <typename E> struct Out {
    static __device__ __forceinline__ void store4(void *out, int64_t at, const float *v)
    {
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(E::pack(v[0], v[1]), E::pack(v[2], v[3]));
    }
};
template <> struct Out<float> {
    static __device__ __forceinline__ void store4(void *out, int64_t at, const float *v)
    {
        *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = make_float4(v[0], v[1], v[2], v[3]);
    }
};

// Row `in_tile` of a tile of rows; called by whole waves.
template <typename E, int D, int ROWS> __device__ __forceinline__ void join_row(const AttendArgs &a, const Item &it, const Seq &s, int kv_head, int in_tile)
{
    constexpr int LANES = D / 4, PARTS = 64 / LANES;  // lanes of a part's row, parts per load
    const int l = lane_id(), row = it.tile * ROWS + in_tile;
    if (row >= s.rows || part_of(a, it, kv_head, it.n_splits - 1) >= a.most_parts)
        return;
    const float *const ml = a.part + (int64_t)a.most_parts * a.rows_cap * D;
    const int token = row / a.group, head = kv_head * a.group + row - token * a.group;
    auto at = [&](int p) __attribute__((always_inline)) { return (int64_t)part_of(a, it, kv_head, p) * a.rows_cap + in_tile; };

    float m = -INFINITY;
    for (int p0 = 0; p0 < it.n_splits; p0 += 64)
        if (p0 + l < it.n_splits)
            m = fmaxf(m, ml[at(p0 + l) * 2]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        m = fmaxf(m, read_from(m, l ^ d));
    float v[4] = {0.f, 0.f, 0.f, 0.f}, weight = 0.f;
    int undefined = 0;
    for (int p0 = 0; p0 < it.n_splits; p0 += 64) {
        const int n = it.n_splits - p0 < 64 ? it.n_splits - p0 : 64;
        JoinedRow j;
        j.m = m;
        float factor = 0.f;  // of part p0 + l
        if (l < n) {
            const float2 x = *reinterpret_cast<const float2 *>(ml + at(p0 + l) * 2);
            factor = j.add_weight(x.x, x.y, a.scale_log2);
        }
        weight += j.w;
        undefined |= (int)j.undefined;
        for (int p1 = 0; p1 < n; p1 += PARTS * kJoinAhead) {
            float4 x[kJoinAhead];
#pragma unroll
            for (int u = 0; u < kJoinAhead; ++u) {
                const int p = p1 + u * PARTS + l / LANES;
                x[u] = *reinterpret_cast<const float4 *>(a.part + at(p0 + (p < n ? p : n - 1)) * D + 4 * (l % LANES));
            }
#pragma unroll
            for (int u = 0; u < kJoinAhead; ++u) {
                const int p = p1 + u * PARTS + l / LANES;
                const float f = read_from(factor, p < n ? p : 0);
                if (p < n && f != 0.f)
                    v[0] += f * x[u].x, v[1] += f * x[u].y, v[2] += f * x[u].z, v[3] += f * x[u].w;
            }
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        weight += read_from(weight, l ^ d);
        undefined |= read_from(undefined, l ^ d);
    }
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] += read_from(v[e], l ^ d);
    JoinedRow j;
    j.m = m, j.w = weight, j.undefined = undefined != 0;
    const float scale = j.scale();
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] *= scale;
    if (l < LANES)
        Out<E>::store4(a.out, (int64_t)(s.start + token) * a.out_stride + (int64_t)head * D + 4 * l, v);
    if (a.lse && l == 0)
        a.lse[(int64_t)(s.start + token) * a.Hq + head] = row_lse<E>(j.m, j.weight(), a.scale_log2);
}

// `rows` rows at a time, `blocks` times per (tile, key head); the workgroups of the launch take them in turn until there are
// no more.  (A workgroup for every piece that there might be took 48 us to find nothing to do for 32768 of them.)
template <typename E, int D, int ROWS, int KT> __global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(AttendArgs a, int rows, int blocks, int workgroups, int most_units)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    for (int unit = blockIdx.x; unit < most_units; unit += workgroups) {
        Item it;
        if (!find_item<ROWS, KT>(a, unit / a.Hkv / blocks, true, &it))
            return;
        const Seq s = load_seq(a, it.seq);
        // key heads fastest, as in the kernels in front: a head's parts are read on the die that wrote them if 8 divide the heads
        for (int r = wave; r < rows; r += kJoinThreads / 64)
            join_row<E, D, ROWS>(a, it, s, unit % a.Hkv, unit / a.Hkv % blocks * rows + r);
    }
}

// ---------------------------------------------------------------- launches
// Rows per tile, workgroups, room for partial results.
struct Launch {
    int rows;             // per tile
    uint32_t target;
    int min_steps, half_steps;
    int64_t most_tiles;   // of all sequences, per key head
    int64_t grid, join_grid, join_units, join_rows, join_blocks, parts, rows_cap;
    size_t bytes;         // of workspace
};
Launch make_launch(const attn_shape_t &s, int batch, int64_t T, int rows, uint32_t target, int min_steps, int half_steps)
{
    Launch c;
    const int64_t group = s.n_q_heads / s.n_kv_heads, all_rows = T * group, seqs = batch < T ? batch : T;
    c.rows = rows;
    c.target = ATTN_TARGET ? (uint32_t)(ATTN_TARGET) : target;
    c.min_steps = ATTN_TARGET ? 1 : min_steps;
    c.half_steps = ATTN_TARGET ? 0 : half_steps;
    c.most_tiles = all_rows / rows + seqs;
    // A tile of a sequence of n steps has at most n / per + 1 / 2 splits, and the sum of n / per over the tiles is at most the target.
    // Only sequences with n >= 3 per / 2 are split.
    c.grid = ((c.target + s.n_kv_heads - 1) / s.n_kv_heads + c.most_tiles) * s.n_kv_heads;
    c.parts = 2 * (int64_t)c.target;
    c.rows_cap = rows < all_rows ? rows : all_rows;
    const int64_t split_tiles = c.most_tiles * s.n_kv_heads < c.target ? c.most_tiles * s.n_kv_heads : c.target;
    // few rows: all at once (32 requests of one token with a single key head 32 us, eight by eight 38); many: fewer look-ups of who
    // they are (2 requests of 100 and 300 tokens 41 us, four by four 44; but the chat turn 32, 31)
    c.join_rows = c.rows_cap <= 16 ? 4 : 8;
    c.join_blocks = (c.rows_cap + c.join_rows - 1) / c.join_rows;
    c.join_units = (split_tiles + s.n_kv_heads - 1) / s.n_kv_heads * s.n_kv_heads * c.join_blocks;
    c.join_grid = c.join_units < kJoinWorkgroups ? c.join_units : kJoinWorkgroups;
    // Where there is a tile for every workgroup that is wanted, only tiles of far more steps than the others are cut: hardly anything to
    // join as a rule, and a few workgroups find that out sooner (256 requests of one token with a window 149 us, by 2048 153; 16
    // packed prompts 306, 309; but where most tiles are cut 64 requests of one token 143, 136).
    if (c.most_tiles * s.n_kv_heads >= c.target && c.join_grid > 256)
        c.join_grid = 256;
    c.bytes = (size_t)(c.parts * c.rows_cap) * (s.head_dim + 2) * sizeof(float);
    return c;
}

// The most steps of KT keys that a tile of `rows` rows can have in a table of this width: fewer than one and a half times
// min_steps are never split.
template <int KT> bool may_split(const AttendArgs &a, const Launch &c)
{
    int64_t steps = ((((int64_t)a.max_blocks << a.log2_bs) + KT - 1) / KT);
    if (a.window > 0) {
        const int64_t seen = ((int64_t)a.window + (a.words > 0 ? 32 * a.words : c.rows / a.group) + 1) / KT + 2 + ((int64_t)a.sinks + KT - 1) / KT;
        steps = seen < steps ? seen : steps;
    }
    return steps + c.min_steps / 2 >= 2 * (int64_t)c.min_steps;
}

template <typename K> hipError_t lds_limit(K kernel, size_t lds)
{
    return lds > 65536 ? hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)
                       : hipSuccess;
}

template <typename K> hipError_t launch_on(K kernel, const AttendArgs &a, const Launch &c, int threads, size_t lds, hipStream_t stream)
{
    const hipError_t e = lds_limit(kernel, lds);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)c.grid), dim3(threads), lds, stream, a);
    return hipGetLastError();
}

AttendArgs attend_args(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, const void *q, int64_t q_stride, const void *k_cache, const void *v_cache,
                       const int32_t *table, const int32_t *cu, const int32_t *cached, float scale, int window, int sinks, void *out, int64_t out_stride, float *lse,
                       void *workspace, const Launch &u)
{
    AttendArgs a;
    a.q = q;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.table = table;
    a.cu = cu;
    a.cached = cached;
    a.out = out;
    a.lse = lse;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.T = T;
    a.batch = batch;
    a.Hq = s.n_q_heads;
    a.Hkv = s.n_kv_heads;
    a.group = s.n_q_heads / s.n_kv_heads;
    a.log2_bs = __builtin_ctz((unsigned)s.block_size);
    a.max_blocks = max_blocks;
    a.n_blocks = n_blocks;
    a.window = window < kMostWindow ? window : kMostWindow;
    a.sinks = sinks;
    a.scale_log2 = scale * kLog2e;
    // finite for the smallest scales as well: added to a maximum of minus infinity it stays minus infinity
    a.outgrown = fminf(kOutgrown / a.scale_log2, FLT_MAX);
    a.part = static_cast<float *>(workspace);
    a.rows_cap = (int)u.rows_cap;
    a.most_parts = (int)u.parts;
    a.target = u.target;
    a.min_steps = u.min_steps;
    a.half_steps = u.half_steps;
    a.positions = a.seen = nullptr;
    a.words = 0;
    return a;
}

}  // namespace
