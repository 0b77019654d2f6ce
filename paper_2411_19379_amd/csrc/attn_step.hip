// Blocks, slots and positions of a step's new tokens, and the append of a layer's keys and values to the paged cache with
// rotary positions on q and k.
#include "attn_common.h"

namespace {

// ---------------------------------------------------------------- blocks, slots, positions
// need_b = ceil((cached_b + n_b) / bs) - ceil(cached_b / bs), one more where a shared block that is not full is replaced, without
// entries behind the end of the table's row; the blocks of sequence b start at the sum of the needs in front of it.  Every
// workgroup computes these sums for itself (a batch is a few KiB of lengths), then the workgroups deal with disjoint tokens and
// disjoint rows of the table.  Small calls are all latency: one launch, and what a workgroup reads of global memory are the
// lengths and, per token, one table entry or one free block (a chat turn 8 us per call, 2.9 of them in the kernel).  A thread's
// four tokens are worked on one after the other, each a search, its sequence's lengths and a table entry that wait for one another:
// 256 requests of up to 512 tokens take the kernel 7.4 us with 21 workgroups for the tokens.  A call hides that behind its 8 us on
// the host, a captured step does not.
constexpr int kAssignThreads = 256;
constexpr int kAssignTokens = 4;  // per thread

struct AssignArgs {
    const int32_t *cu, *cached, *shared, *table_in, *free_blocks, *n_free;
    int32_t *table_out, *positions, *copies, *counts;
    int64_t *slots;
    int64_t T;
    int32_t batch, log2_bs, max_blocks, free_capacity;
    int32_t token_workgroups, table_workgroups;  // the first ones deal with tokens, the others with rows of the table
};

struct AssignSeq {
    int start, n, cached;
    int have;   // table entries that stay
    int all;    // entries with the new tokens
    bool fork;  // the last cached block is replaced
    // entries that want a block, of those that the row has
    __device__ __forceinline__ int need(int max_blocks) const
    {
        const int end = all < max_blocks ? all : max_blocks;
        return n > 0 && end > have ? end - have : 0;
    }
    // entries of new tokens that the row does not have
    __device__ __forceinline__ int behind(const AssignArgs &a) const
    {
        const int first = cached >> a.log2_bs;
        const int from = first > a.max_blocks ? first : a.max_blocks;
        return n > 0 && all > from ? all - from : 0;
    }
};
__device__ __forceinline__ AssignSeq assign_seq(const AssignArgs &a, int b)
{
    AssignSeq s;
    const int bs = 1 << a.log2_bs;
    const int64_t from = a.cu[b] < 0 ? 0 : a.cu[b], to = a.cu[b + 1] > a.T ? a.T : a.cu[b + 1];
    s.start = (int)from;
    s.n = to > from ? (int)(to - from) : 0;
    const int c = a.cached[b];
    s.cached = c < 0 ? 0 : c > 0x3fffffff ? 0x3fffffff : c;
    s.fork = s.n > 0 && a.shared && a.shared[b] != 0 && (s.cached & (bs - 1)) != 0;
    s.have = (int)(((int64_t)s.cached + bs - 1) >> a.log2_bs) - (s.fork ? 1 : 0);
    s.all = (int)(((int64_t)s.cached + s.n + bs - 1) >> a.log2_bs);
    return s;
}
// The order-th block that the call hands out.
__device__ __forceinline__ int free_block(const AssignArgs &a, int n_free, int64_t order)
{
    return (uint64_t)order < (uint64_t)n_free ? a.free_blocks[n_free - 1 - order] : -1;
}
// Sums of needs take 64 bits: the needs of sequences that name the same tokens again and again exceed 32.  wave_scan of values up
// to 2^31, in halves of 16 bits, whose sums over a wave fit.
__device__ __forceinline__ int64_t wave_scan64(int v) { return ((int64_t)wave_scan(v >> 16) << 16) + wave_scan(v & 0xffff); }
__device__ __forceinline__ int sat32(int64_t v) { return v > 0x7fffffff ? 0x7fffffff : (int)v; }

__global__ __launch_bounds__(kAssignThreads) void attn_assign_kernel(AssignArgs a)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    int *start = reinterpret_cast<int *>(lds_raw);        // [batch] first token of each sequence
    int *base = start + a.batch;                          // [batch] blocks handed out in front of it, 2^31 - 1 if more
    int64_t *sums = reinterpret_cast<int64_t *>(base + a.batch);  // [4]
    uint32_t *behind_sums = reinterpret_cast<uint32_t *>(sums + kAssignThreads / 64);  // [4]
    const int tid = threadIdx.x, wave = tid / 64, l = lane_id();
    int n_free = *a.n_free;
    n_free = n_free < 0 ? 0 : n_free > a.free_capacity ? a.free_capacity : n_free;
    int64_t before = 0;
    uint32_t behind = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kAssignThreads) {
        const int b = b0 + tid;
        int need = 0;
        if (b < a.batch) {
            const AssignSeq s = assign_seq(a, b);
            need = s.need(a.max_blocks);
            behind = sat_add(behind, (uint32_t)s.behind(a));
            start[b] = s.start;
        }
        const int64_t upto = wave_scan64(need);
        lds_barrier();
        if (l == 63)
            sums[wave] = upto;
        lds_barrier();
        int64_t mine = before + upto - need;
        for (int w = 0; w < kAssignThreads / 64; ++w) {
            mine += w < wave ? sums[w] : 0;
            before += sums[w];
        }
        if (b < a.batch)
            base[b] = sat32(mine);
    }
    behind = wave_sat_sum(behind);
    if (l == 0)
        behind_sums[wave] = behind;
    lds_barrier();
    const int bs = 1 << a.log2_bs;
    if ((int)blockIdx.x < a.token_workgroups) {
        if (blockIdx.x == 0 && tid == 0) {
            a.counts[0] = before < n_free ? (int)(n_free - before) : 0;
            int64_t missing = before > n_free ? before - n_free : 0;
            for (int w = 0; w < kAssignThreads / 64; ++w)
                missing += behind_sums[w];
            a.counts[1] = sat32(missing);
        }
#pragma unroll 1
        for (int u = 0; u < kAssignTokens; ++u) {
            const int64_t t = ((int64_t)blockIdx.x * kAssignTokens + u) * kAssignThreads + tid;
            if (t >= a.T)
                return;
            int lo = 0, hi = a.batch;  // the last sequence that starts at t or in front of it
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                (start[mid] <= t ? lo : hi) = mid;
            }
            const AssignSeq s = assign_seq(a, lo);
            int64_t slot = -1;
            int pos = 0;
            if (t >= s.start && t - s.start < s.n) {
                pos = s.cached + (int)(t - s.start);
                const int e = pos >> a.log2_bs;
                if (e < a.max_blocks) {
                    const int block = e < s.have ? a.table_in[(int64_t)lo * a.max_blocks + e] : free_block(a, n_free, (int64_t)base[lo] + e - s.have);
                    slot = block < 0 ? -1 : ((int64_t)block << a.log2_bs) + (pos & (bs - 1));
                }
            }
            a.slots[t] = slot;
            a.positions[t] = pos;
        }
        return;
    }
    const bool in_place = a.table_in == a.table_out;
    for (int b = blockIdx.x - a.token_workgroups; b < a.batch; b += a.table_workgroups) {
        const AssignSeq s = assign_seq(a, b);
        const int32_t *in = a.table_in + (int64_t)b * a.max_blocks;
        int32_t *out = a.table_out + (int64_t)b * a.max_blocks;
        if (tid == 0) {  // in front of the entry's replacement by the same thread
            int from = -1, to = -1, rows = 0;
            if (s.fork && s.have < a.max_blocks) {
                from = in[s.have];
                to = free_block(a, n_free, base[b]);
                rows = s.cached & (bs - 1);
                out[s.have] = to;
            }
            int32_t *c = a.copies + (int64_t)b * 4;
            c[0] = from, c[1] = to, c[2] = rows, c[3] = 0;
        }
        const int first_new = s.have + (s.fork ? 1 : 0), all = s.n > 0 ? s.all : s.have;
        for (int e = (in_place ? first_new : 0) + tid; e < (in_place ? (all < a.max_blocks ? all : a.max_blocks) : a.max_blocks);
             e += kAssignThreads) {
            if (s.fork && e == s.have)
                continue;
            out[e] = e < s.have ? in[e] : e < all ? free_block(a, n_free, (int64_t)base[b] + e - s.have) : -1;
        }
    }
}

// ---------------------------------------------------------------- rotary positions and the append
// Streaming: every value of q, k and v is read and written once.  A thread takes 8 values of v, or of a part of a head that
// does not turn, or 8 pairs of a head of q or k (two runs of 8 values in the half layout, one of 16 interleaved).  Memory bounds
// it: 32768 tokens of 32 + 8 + 8 heads of 128 in bf16 142 us, 5.8 TB/s; small calls are a launch (64 tokens 8 us, the kernel 3).
constexpr int kRopeThreads = 256;

struct RopeArgs {
    const void *q, *k, *v;
    void *q_out, *k_cache, *v_cache;
    const int32_t *positions, *copies;
    const int64_t *slots;
    const float *rotary;
    int64_t q_stride, k_stride, v_stride, T;
    int64_t n_slots;
    int32_t Hq, Hkv, D, log2_bs, n_blocks, max_positions, rot;
    int32_t turned_units, head_units, token_units;  // of a head of q or k: pair units, all units; of a token
    int64_t token_workgroups;
    int32_t interleaved;
};

// 8 neighbouring values
template <typename E> struct Eight {
    typedef uint16_t type;
    static __device__ __forceinline__ void read(const uint16_t *p, float *v)
    {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        v[0] = E::lo(a.x), v[1] = E::hi(a.x), v[2] = E::lo(a.y), v[3] = E::hi(a.y);
        v[4] = E::lo(a.z), v[5] = E::hi(a.z), v[6] = E::lo(a.w), v[7] = E::hi(a.w);
    }
    static __device__ __forceinline__ void write(uint16_t *p, const float *v)
    {
        *reinterpret_cast<uint4 *>(p) = make_uint4(E::pack(v[0], v[1]), E::pack(v[2], v[3]), E::pack(v[4], v[5]), E::pack(v[6], v[7]));
    }
    static __device__ __forceinline__ void copy(const uint16_t *from, uint16_t *to) { *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from); }
};
template <> struct Eight<float> {
    typedef float type;
    static __device__ __forceinline__ void read(const float *p, float *v)
    {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    static __device__ __forceinline__ void write(float *p, const float *v)
    {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
    static __device__ __forceinline__ void copy(const float *from, float *to)
    {
        const uint4 a = reinterpret_cast<const uint4 *>(from)[0], b = reinterpret_cast<const uint4 *>(from)[1];
        reinterpret_cast<uint4 *>(to)[0] = a;
        reinterpret_cast<uint4 *>(to)[1] = b;
    }
};

template <typename E> __global__ __launch_bounds__(kRopeThreads) void attn_rope_kernel(RopeArgs a)
{
    typedef Eight<E> V;
    typedef typename V::type elem;
    const int bs = 1 << a.log2_bs;
    if ((int64_t)blockIdx.x >= a.token_workgroups) {
        // the shared tail blocks: a workgroup per sequence, cache and head, whose rows are contiguous (a workgroup per sequence
        // took 15 us for 15 rows of 4 heads)
        const int unit = (int)(blockIdx.x - a.token_workgroups), of_seq = 2 * a.Hkv, seq = unit / of_seq, h = (unit - seq * of_seq) >> 1;
        const int32_t *c = a.copies + (int64_t)seq * 4;
        const int from = c[0], to = c[1], rows = c[2] < bs ? c[2] : bs;
        if ((uint32_t)from >= (uint32_t)a.n_blocks || (uint32_t)to >= (uint32_t)a.n_blocks)
            return;
        elem *const cache = static_cast<elem *>(unit & 1 ? a.v_cache : a.k_cache);
        const elem *const src = cache + (((int64_t)from * a.Hkv + h) << a.log2_bs) * a.D;
        elem *const dst = cache + (((int64_t)to * a.Hkv + h) << a.log2_bs) * a.D;
        for (int i = threadIdx.x; i < rows * (a.D / 8); i += kRopeThreads)
            V::copy(src + i * 8, dst + i * 8);
        return;
    }
    const int64_t at = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    const int64_t t = at / a.token_units;
    int unit = (int)(at - t * a.token_units);
    if (t >= a.T)
        return;
    const int turning = (a.Hq + a.Hkv) * a.head_units;
    const bool of_v = unit >= turning;
    const int per_head = of_v ? a.D / 8 : a.head_units;
    unit -= of_v ? turning : 0;
    int head = unit / per_head;
    const int part = unit - head * per_head;
    const bool of_q = !of_v && head < a.Hq;
    head -= of_v || of_q ? 0 : a.Hq;
    const elem *src = static_cast<const elem *>(of_v ? a.v : of_q ? a.q : a.k) + t * (of_v ? a.v_stride : of_q ? a.q_stride : a.k_stride) +
                      (int64_t)head * a.D;
    elem *dst;
    if (of_q) {
        dst = static_cast<elem *>(a.q_out) + (t * a.Hq + head) * a.D;
    } else {
        const int64_t slot = a.slots[t];
        if (slot < 0 || slot >= a.n_slots)
            return;
        dst = static_cast<elem *>(of_v ? a.v_cache : a.k_cache) +
              (((((slot >> a.log2_bs) * a.Hkv + head) << a.log2_bs) + (slot & (bs - 1))) * a.D);
    }
    if (of_v || part >= a.turned_units) {
        const int d = of_v ? part * 8 : a.rot + (part - a.turned_units) * 8;
        V::copy(src + d, dst + d);
        return;
    }
    const int d0 = a.interleaved ? part * 16 : part * 8, d1 = a.interleaved ? d0 + 8 : d0 + a.rot / 2;
    const int pos = a.positions[t];
    const bool known = (uint32_t)pos < (uint32_t)a.max_positions;
    float c[8], s[8], x[8], y[8];
    const float *const row = a.rotary + (int64_t)(known ? pos : 0) * a.rot + part * 8;
    Eight<float>::read(row, c);
    Eight<float>::read(row + a.rot / 2, s);
    V::read(src + d0, x);
    V::read(src + d1, y);
    const float nan_else_0 = known ? 0.f : NAN;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        c[e] += nan_else_0, s[e] += nan_else_0;
    float u[8], v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        // interleaved: x and y hold pairs 0..3 and 4..7
        const float first = a.interleaved ? (e < 4 ? x : y)[2 * (e % 4)] : x[e], second = a.interleaved ? (e < 4 ? x : y)[2 * (e % 4) + 1] : y[e];
        u[e] = first * c[e] - second * s[e];
        v[e] = second * c[e] + first * s[e];
    }
    float p[8], q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        p[e] = a.interleaved ? (e % 2 ? v : u)[e / 2] : u[e];
        q[e] = a.interleaved ? (e % 2 ? v : u)[4 + e / 2] : v[e];
    }
    V::write(dst + d0, p);
    V::write(dst + d1, q);
}

}  // namespace

hipError_t launch_attn_assign(int batch, int log2_bs, int max_blocks, int64_t T, const int32_t *cu, const int32_t *cached,
                              const int32_t *shared, const int32_t *table_in, int32_t *table_out, const int32_t *free_blocks,
                              const int32_t *n_free, int32_t free_capacity, int64_t *slots, int32_t *positions, int32_t *copies,
                              int32_t *counts, hipStream_t stream)
{
    AssignArgs a;
    a.cu = cu;
    a.cached = cached;
    a.shared = shared;
    a.table_in = table_in;
    a.free_blocks = free_blocks;
    a.n_free = n_free;
    a.table_out = table_out;
    a.positions = positions;
    a.copies = copies;
    a.counts = counts;
    a.slots = slots;
    a.T = T;
    a.batch = batch;
    a.log2_bs = log2_bs;
    a.max_blocks = max_blocks;
    a.free_capacity = free_capacity;
    const int64_t per = kAssignThreads * kAssignTokens;
    a.token_workgroups = (int)(T > 0 ? (T + per - 1) / per : 1);  // the first one also writes the counts
    a.table_workgroups = batch < 256 ? batch : 256;
    const size_t lds = 2 * (size_t)batch * sizeof(int) + kAssignThreads / 64 * (sizeof(int64_t) + sizeof(uint32_t));
    hipLaunchKernelGGL(attn_assign_kernel, dim3((unsigned)(a.token_workgroups + a.table_workgroups)), dim3(kAssignThreads), lds,
                       stream, a);
    return hipGetLastError();
}

hipError_t launch_attn_rope(const attn_shape_t &s, int64_t T, int batch, int n_blocks, const void *q, int64_t q_stride,
                            const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *positions,
                            const int64_t *slots, const float *rotary, int max_positions, int rotary_dim, bool interleaved,
                            const int32_t *copies, void *q_out, void *k_cache, void *v_cache, hipStream_t stream)
{
    RopeArgs a;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_out = q_out;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.positions = positions;
    a.copies = copies;
    a.slots = slots;
    a.rotary = rotary;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.T = T;
    a.Hq = s.n_q_heads;
    a.Hkv = s.n_kv_heads;
    a.D = s.head_dim;
    a.log2_bs = __builtin_ctz((unsigned)s.block_size);
    a.n_blocks = n_blocks;
    a.n_slots = (int64_t)n_blocks << a.log2_bs;
    a.max_positions = max_positions;
    a.rot = rotary_dim;
    a.turned_units = rotary_dim / 16;
    a.head_units = rotary_dim / 16 + (s.head_dim - rotary_dim) / 8;
    a.token_units = (a.Hq + a.Hkv) * a.head_units + a.Hkv * (a.D / 8);
    a.interleaved = interleaved;
    a.token_workgroups = (T * a.token_units + kRopeThreads - 1) / kRopeThreads;
    const int64_t n = a.token_workgroups + (copies ? (int64_t)batch * 2 * a.Hkv : 0);
    if (n == 0)
        return hipSuccess;
    if (n > 0x7fffffff)
        return hipErrorInvalidValue;
    const dim3 grid((unsigned)n), block(kRopeThreads);
    if (s.io_dtype == ATTN_DT_F32)
        hipLaunchKernelGGL((attn_rope_kernel<float>), grid, block, 0, stream, a);
    else if (s.io_dtype == ATTN_DT_BF16)
        hipLaunchKernelGGL((attn_rope_kernel<Bf16>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((attn_rope_kernel<F16>), grid, block, 0, stream, a);
    return hipGetLastError();
}
