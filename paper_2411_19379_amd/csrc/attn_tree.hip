// What a step that checks trees of drafted tokens does beside the attention: positions and visibility of the tokens, the branch that
// the model agrees with, and its keys and values to where a chain of tokens has them.
#include "attn_common.h"

namespace {

struct TreeSeq {
    int start, n, cached;
};
__device__ __forceinline__ TreeSeq tree_seq(const int32_t *cu, const int32_t *cached, int b, int64_t T)
{
    TreeSeq s;
    const int from = cu[b] < 0 ? 0 : cu[b], to = cu[b + 1] > T ? (int)T : cu[b + 1], c = cached[b];
    s.start = from;
    s.n = to > from ? to - from : 0;
    s.cached = c < 0 ? 0 : c > 0x3fffffff ? 0x3fffffff : c;
    return s;
}

// ---------------------------------------------------------------- positions and visibility
// depth(i) = depth(p(i)) + 1, position = cached + depth;  seen(i) = {i} u seen(p(i)), of which a window leaves the near ones and the
// sinks.  A workgroup per sequence, its parents in LDS, a thread per token that walks up to the root: ancestors come in falling
// order, so a thread has one word of its bits in hand at a time.  All latency: the lengths, the parents, a walk of some 100 cycles
// per ancestor, with a window a second one in front that counts them.
constexpr int kDraftThreads = 256;

__global__ __launch_bounds__(kDraftThreads) void attn_draft_tree_kernel(int batch, int64_t T, int words, const int32_t *parents, const int32_t *cu,
                                                                       const int32_t *cached, int window, int sinks, int32_t *positions,
                                                                       int32_t *seen)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    int *const parent = reinterpret_cast<int *>(lds_raw);  // [32 words]
    const int tid = threadIdx.x;
    if ((int)blockIdx.x == batch) {  // tokens of no sequence
        const int first = cu[0] > 0 ? cu[0] : 0, last = cu[batch] < 0 ? 0 : cu[batch];
        auto clear = [&](int64_t from, int64_t to) __attribute__((always_inline)) {
            for (int64_t t = from + tid; t < to; t += kDraftThreads)
                positions[t] = 0;
            for (int64_t k = from * words + tid; k < to * words; k += kDraftThreads)
                seen[k] = 0;
        };
        clear(0, first < T ? first : T);
        clear(last < first ? first : last, T);
        return;
    }
    const TreeSeq s = tree_seq(cu, cached, blockIdx.x, T);
    const int most = 32 * words, n = s.n < most ? s.n : most;
    for (int i = tid; i < n; i += kDraftThreads) {
        const int p = parents[s.start + i];
        parent[i] = p >= 0 && p < i ? p : -1;
    }
    lds_barrier();
    for (int i = tid; i < s.n; i += kDraftThreads) {
        int32_t *const row = seen + (int64_t)(s.start + i) * words;
        if (i >= n) {  // no bit for it
            positions[s.start + i] = s.cached;
            for (int w = 0; w < words; ++w)
                row[w] = 0;
            continue;
        }
        int depth = 0;
        if (window > 0)
            for (int a = parent[i]; a >= 0; a = parent[a])
                ++depth;
        int word = i >> 5, steps = 0;
        uint32_t bits = 0;
        for (int w = words - 1; w > word; --w)
            row[w] = 0;
        for (int a = i; a >= 0; a = parent[a], ++steps) {
            for (; word > a >> 5; --word, bits = 0)
                row[word] = (int32_t)bits;
            if (window <= 0 || steps < window || s.cached + depth - steps < sinks)
                bits |= 1u << (a & 31);
        }
        for (; word >= 0; --word, bits = 0)
            row[word] = (int32_t)bits;
        positions[s.start + i] = s.cached + steps - 1;
    }
}

// ---------------------------------------------------------------- the branch that is kept
// v_0 is the sequence's first token, v_(k+1) the first child of v_k that is the token chosen behind v_k.  A wave per sequence, a token
// per lane and 64 at a time: children come behind their parents, so one walk over the tokens finds the branch.  One workgroup for the
// batch, since the blocks that are given back go to the free list in the order of the sequences and their places are a sum over those
// in front (the walks would not need it: every further 64 trees are one more pass); a wave has the tokens of up to kAcceptAtOnce
// sequences on their way at once.  Latency bounds it: a launch, four trips to memory and two barriers; one tree 4.5 us, 64 trees of 16
// to 64 tokens 12 us (walking four sequences side by side, with the blocks kept in registers, 11.7).
constexpr int kAcceptThreads = 1024;
constexpr int kAcceptWaves = kAcceptThreads / 64;
constexpr int kAcceptAtOnce = 4;

struct AcceptArgs {
    const int32_t *tokens, *parents, *choices, *cu, *cached, *table, *n_free;
    int32_t *free_blocks, *path, *counts, *next_tokens, *kept_lens, *n_free_out;
    int64_t T;
    int32_t batch, log2_bs, max_blocks, free_capacity;
};
// Entries of the table's row that hold only tokens that are not kept.
__device__ __forceinline__ void given_back(const AcceptArgs &a, const TreeSeq &s, int count, int *first, int *last)
{
    const int bs = 1 << a.log2_bs;
    const int all = (int)(((int64_t)s.cached + s.n + bs - 1) >> a.log2_bs);
    *first = (int)(((int64_t)s.cached + count + bs - 1) >> a.log2_bs);
    *last = all < a.max_blocks ? all : a.max_blocks;
}

__global__ __launch_bounds__(kAcceptThreads) void attn_accept_kernel(AcceptArgs a)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    int *const counts = reinterpret_cast<int *>(lds_raw);                          // [batch] kept tokens
    int *const back = counts + a.batch;                                            // [batch] blocks given back, then those in front
    int64_t *const sums = reinterpret_cast<int64_t *>(lds_raw + ((size_t)a.batch * 8 + 15) / 16 * 16);  // [waves]
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = lane_id();
    {  // tokens of no sequence
        const int first = a.cu[0] > 0 ? a.cu[0] : 0, last = a.cu[a.batch] < 0 ? 0 : a.cu[a.batch];
        for (int64_t t = tid; t < first && t < a.T; t += kAcceptThreads)
            a.path[t] = -1;
        for (int64_t t = last + (int64_t)tid; t < a.T; t += kAcceptThreads)
            a.path[t] = -1;
    }
    for (int b0 = 0; b0 < a.batch; b0 += kAcceptWaves * kAcceptAtOnce) {
        TreeSeq s[kAcceptAtOnce];
        int token[kAcceptAtOnce], parent[kAcceptAtOnce], choice[kAcceptAtOnce];
#pragma unroll
        for (int u = 0; u < kAcceptAtOnce; ++u) {
            const int b = b0 + u * kAcceptWaves + wave;
            s[u] = tree_seq(a.cu, a.cached, b < a.batch ? b : a.batch - 1, a.T);
            s[u].n = b < a.batch ? s[u].n : 0;
        }
        auto load = [&](int u, int first) __attribute__((always_inline)) {
            const bool there = first + l < s[u].n;
            const int64_t t = s[u].start + (int64_t)(there ? first + l : 0);
            token[u] = there ? a.tokens[t] : 0;
            parent[u] = there ? a.parents[t] : -2;  // no token's child
            choice[u] = there ? a.choices[t] : -1;
        };
#pragma unroll
        for (int u = 0; u < kAcceptAtOnce; ++u)
            load(u, 0);
#pragma unroll
        for (int u = 0; u < kAcceptAtOnce; ++u) {
            const int b = b0 + u * kAcceptWaves + wave;
            if (b >= a.batch)
                continue;
            const int n = s[u].n;
            int count = 0, at = -1, chosen = -1;
            for (int first = 0; first < n; first += 64) {
                if (first > 0)
                    load(u, first);
                uint64_t kept = 0;
                if (first == 0) {
                    at = 0, chosen = __builtin_amdgcn_readlane(choice[u], 0), kept = 1;
                }
                for (;;) {
                    const int here = at - first;  // children lie behind it
                    const uint64_t child = __ballot(parent[u] == at && token[u] == chosen && l > here);
                    if (child == 0)
                        break;
                    const int c = __builtin_ctzll(child);
                    kept |= 1ull << c;
                    at = first + c;
                    chosen = __builtin_amdgcn_readlane(choice[u], c);
                }
                if (kept >> l & 1)
                    a.path[s[u].start + (int64_t)(count + __popcll(kept & first_bits(l)))] = first + l;
                count += __popcll(kept);
            }
            for (int64_t k = count + l; k < n; k += 64)
                a.path[s[u].start + k] = -1;
            if (l == 0) {
                a.counts[b] = count;
                a.next_tokens[b] = chosen;
                a.kept_lens[b] = s[u].cached + count;
                counts[b] = count;
            }
            if (a.table) {
                int e0, e1;
                given_back(a, s[u], count, &e0, &e1);
                uint32_t n_back = 0;
                for (int e = e0; e < e1; e += 64)
                    n_back += (uint32_t)__popcll(__ballot(e + l < e1 && a.table[(int64_t)b * a.max_blocks + (e + l < e1 ? e + l : e)] >= 0));
                if (l == 0)
                    back[b] = (int)n_back;
            }
        }
    }
    if (!a.table)
        return;
    lds_barrier();
    int n_free = *a.n_free;
    n_free = n_free < 0 ? 0 : n_free > a.free_capacity ? a.free_capacity : n_free;
    int64_t before = n_free;
    for (int b0 = 0; b0 < a.batch; b0 += kAcceptThreads) {
        const int b = b0 + tid, mine = b < a.batch ? back[b] : 0;
        // sums over a wave may exceed 32 bits: in halves of 16
        const int64_t upto = ((int64_t)wave_scan(mine >> 16) << 16) + wave_scan(mine & 0xffff);
        lds_barrier();
        if (l == 63)
            sums[wave] = upto;
        lds_barrier();
        int64_t in_front = before + upto - mine;
        for (int w = 0; w < kAcceptWaves; ++w) {
            in_front += w < wave ? sums[w] : 0;
            before += sums[w];
        }
        if (b < a.batch)
            back[b] = in_front > a.free_capacity ? a.free_capacity : (int)in_front;
    }
    if (tid == 0)
        *a.n_free_out = before > a.free_capacity ? a.free_capacity : (int)before;
    lds_barrier();
    for (int b = wave; b < a.batch; b += kAcceptWaves) {
        const TreeSeq s = tree_seq(a.cu, a.cached, b, a.T);
        int e0, e1, to = back[b];
        given_back(a, s, counts[b], &e0, &e1);
        for (int e = e0; e < e1 && to < a.free_capacity; e += 64) {
            const int id = e + l < e1 ? a.table[(int64_t)b * a.max_blocks + e + l] : -1;
            const uint64_t valid = __ballot(id >= 0);
            const int64_t at = (int64_t)to + __popcll(valid & first_bits(l));
            if (id >= 0 && at < a.free_capacity)
                a.free_blocks[at] = id;
            to += __popcll(valid);
        }
    }
}

// ---------------------------------------------------------------- keys and values of the branch
// Row cached + path[k] of every cache goes to row cached + k.  path[k] >= k and rises, so in rising order no row is overwritten
// before it has been read; a thread has the same 16 bytes of all rows and keeps that order.  Where the rows lie is looked up by a lane
// per kept token, 64 at once: lengths, path and table are three trips to memory (with every thread looking up its rows, eight at a
// time, 64 trees and 16 caches took 8.9 us, so 5.7).  Rows are written as kKeepAtOnce at a time, but the compiler keeps them in
// scratch memory, 144 bytes per lane, as their loads are in branches: each is waited for, written there and read back.
constexpr int kKeepThreads = 256;
constexpr int kKeepAtOnce = 8;

struct KeepArgs {
    void *caches[kCachesPerLaunch];
    const int32_t *table, *cu, *cached, *path;
    int64_t T;
    int32_t n_caches, Hkv, pieces, log2_bs, max_blocks, n_blocks;
};

__global__ __launch_bounds__(kKeepThreads) void attn_keep_kernel(KeepArgs a)
{
    const int b = blockIdx.y, unit = blockIdx.x * kKeepThreads + threadIdx.x, l = lane_id();
    const int piece = unit % a.pieces, head = unit / a.pieces % a.Hkv, cache = unit / a.pieces / a.Hkv;
    const TreeSeq s = tree_seq(a.cu, a.cached, b, a.T);
    const bool moves_any = cache < a.n_caches;
    uint4 *const base = static_cast<uint4 *>(a.caches[moves_any ? cache : 0]) + piece;
    for (int k0 = 0; k0 < s.n; k0 += 64) {
        const int k = k0 + l, from = k < s.n ? a.path[s.start + (int64_t)k] : -1;
        // the branch ends at the first entry that is none
        const uint64_t valid = __ballot(from >= k && from < s.n);
        const uint64_t kept = valid == ~0ull ? ~0ull : first_bits(__builtin_ctzll(~valid));
        auto slot = [&](int i, int *block, int *row) __attribute__((always_inline)) {  // of new token i
            const int64_t j = (int64_t)s.cached + i, e = j >> a.log2_bs;
            *block = e < a.max_blocks ? a.table[(int64_t)b * a.max_blocks + e] : -1;
            *row = (int)(j & ((1 << a.log2_bs) - 1));
        };
        int from_block = -1, from_row = 0, to_block = -1, to_row = 0;
        if ((kept >> l & 1) != 0 && from > k) {
            slot(from, &from_block, &from_row);
            slot(k, &to_block, &to_row);
        }
        uint64_t left = __ballot((uint32_t)from_block < (uint32_t)a.n_blocks && (uint32_t)to_block < (uint32_t)a.n_blocks);
        while (left != 0) {
            uint4 v[kKeepAtOnce];
            int64_t to[kKeepAtOnce];
#pragma unroll
            for (int u = 0; u < kKeepAtOnce; ++u) {
                to[u] = -1;
                if (left == 0)
                    continue;
                const int lane = __builtin_ctzll(left);
                left &= left - 1;
                auto at = [&](int block, int row) __attribute__((always_inline)) {
                    const int first = __builtin_amdgcn_readlane(block, lane) * a.Hkv;
                    return ((int64_t)(first + head) << a.log2_bs) + __builtin_amdgcn_readlane(row, lane);
                };
                to[u] = at(to_block, to_row) * a.pieces;
                const int64_t source = at(from_block, from_row) * a.pieces;
                if (moves_any)
                    v[u] = base[source];
            }
#pragma unroll
            for (int u = 0; u < kKeepAtOnce; ++u)
                if (to[u] >= 0 && moves_any)
                    base[to[u]] = v[u];
        }
        if (kept != ~0ull)
            return;
    }
}

}  // namespace

hipError_t launch_attn_draft_tree(int batch, int64_t T, int words, const int32_t *parents, const int32_t *cu, const int32_t *cached,
                                  int window, int sinks, int32_t *positions, int32_t *seen, hipStream_t stream)
{
    hipLaunchKernelGGL(attn_draft_tree_kernel, dim3((unsigned)batch + 1), dim3(kDraftThreads), (size_t)words * 32 * sizeof(int), stream, batch, T, words,
                       parents, cu, cached, window, sinks, positions, seen);
    return hipGetLastError();
}

hipError_t launch_attn_accept(int batch, int log2_bs, int max_blocks, int64_t T, const int32_t *tokens, const int32_t *parents,
                              const int32_t *choices, const int32_t *cu, const int32_t *cached, const int32_t *table,
                              int32_t *free_blocks, const int32_t *n_free, int32_t free_capacity, int32_t *path, int32_t *counts,
                              int32_t *next_tokens, int32_t *kept_lens, int32_t *n_free_out, hipStream_t stream)
{
    AcceptArgs a;
    a.tokens = tokens, a.parents = parents, a.choices = choices, a.cu = cu, a.cached = cached, a.table = table, a.n_free = n_free;
    a.free_blocks = free_blocks, a.path = path, a.counts = counts, a.next_tokens = next_tokens, a.kept_lens = kept_lens, a.n_free_out = n_free_out;
    a.T = T, a.batch = batch, a.log2_bs = log2_bs, a.max_blocks = max_blocks, a.free_capacity = free_capacity;
    const size_t lds = ((size_t)batch * 8 + 15) / 16 * 16 + kAcceptWaves * sizeof(int64_t);
    hipLaunchKernelGGL(attn_accept_kernel, dim3(1), dim3(kAcceptThreads), lds, stream, a);
    return hipGetLastError();
}

hipError_t launch_attn_keep(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, int n_caches,
                            void *const *caches, const int32_t *table, const int32_t *cu, const int32_t *cached,
                            const int32_t *path, hipStream_t stream)
{
    KeepArgs a;
    a.table = table, a.cu = cu, a.cached = cached, a.path = path;
    a.T = T, a.Hkv = s.n_kv_heads, a.log2_bs = __builtin_ctz((unsigned)s.block_size), a.max_blocks = max_blocks, a.n_blocks = n_blocks;
    a.pieces = s.head_dim * (s.io_dtype == ATTN_DT_F32 ? 4 : 2) / 16;
    for (int first = 0; first < n_caches; first += kCachesPerLaunch) {
        a.n_caches = n_caches - first < kCachesPerLaunch ? n_caches - first : kCachesPerLaunch;
        for (int c = 0; c < a.n_caches; ++c)
            a.caches[c] = caches[first + c];
        const int units = a.n_caches * a.Hkv * a.pieces;
        hipLaunchKernelGGL(attn_keep_kernel, dim3((unsigned)((units + kKeepThreads - 1) / kKeepThreads), (unsigned)batch), dim3(kKeepThreads), 0, stream, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}
