// The gated recurrence over packed sequences, and its backward pass.
//
// h_t = a_t h_(t-1) + b_t is the composition of maps h -> a h + b, which compose as (A, H) then (A', H') = (A A', A' H + H').  Tokens
// are cut into chunks of 64 for a workgroup and 16 (8 in the backward pass) for a wave; a lane has V channels of all of a wave's
// tokens.  A wave composes its tokens from registers, the workgroup its waves, and the state in front of a chunk comes from the
// workgroups in front of it while the chunk's values wait in registers, so that inputs are read once and gates, which cost as much as
// the reads, are computed once.  Backwards the same with q_t = a_t (dy_t + q_(t+1)), what a state's gradient hands to the one in
// front, over chunks in falling order.
//
// A workgroup takes the number of its chunk from a counter of its channels when it starts: what it waits for is in the hands
// of workgroups that run already, whatever order they are started in, so every wait ends.  A chunk publishes its (A, H) at once;
// the next ones of its group of 16 chunks compose them in order, behind the state that the last chunk of the group in front has
// published.  The order of all sums is fixed by the chunks' numbers.  What is published is one 64-bit word per channel (32-bit for
// a state), which holds a pattern that no result has until it is there: no other memory has to be ordered by it.
#include <cmath>

#include "rec_common.h"

namespace {

constexpr int kChunk = 64;          // tokens
constexpr int kGroup = 16;          // chunks
constexpr uint32_t kNothing = 0xffffffffu;
constexpr int kMostPolls = 1 << 22; // of a wait: seconds; its result is NaN then, and the grid still drains
constexpr float kCut = -1.f;        // A of a map that forgets what was in front: a sequence starts in it

__device__ __forceinline__ float never_nothing(float v) { return v != v ? __uint_as_float(0x7fc00000u) : v; }
// H' of a map (A, H) of `carry`
__device__ __forceinline__ float apply(float A, float H, float carry) { return A < 0.f ? H : __builtin_fmaf(A, carry, H); }

struct Look {
    uint64_t *maps;    // [chunks][channels] of the chunks
    uint32_t *states;  // [groups][channels] behind the groups
    int *tickets;      // [channel blocks]
    float *rate;       // [channels]
    int32_t channels, n_chunks, n_blocks;
};
__device__ __forceinline__ uint64_t load_published(const uint64_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t load_published(const uint32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void publish(uint64_t *p, uint64_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void publish(uint32_t *p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// ---------------------------------------------------------------- in front of a scan
// Nothing is published yet, no chunk is taken; the channels' rates, whose softplus would cost a chunk as much as two of its tokens.
constexpr int kPrepareThreads = 256;
__global__ __launch_bounds__(kPrepareThreads) void rec_prepare_kernel(uint32_t *words, int64_t n_words, int *tickets, int n_tickets, float *rate, const float *decay,
                                                                     float sharpness, int channels, int64_t stride)
{
    const int64_t at = (int64_t)blockIdx.x * kPrepareThreads + threadIdx.x;
    for (int64_t k = at; k < n_words; k += stride)
        words[k] = kNothing;
    for (int64_t k = at; k < n_tickets; k += stride)
        tickets[k] = 0;
    for (int64_t k = at; k < channels; k += stride)
        rate[k] = decay_rate(decay[k], sharpness);
}

// ---------------------------------------------------------------- where sequences begin and end in a chunk
struct Edges {
    int first[kChunk], last[kChunk], ckpt[kChunk];  // sequence + 1 that begins or ends with the token; whether its state is wanted
};
__device__ __forceinline__ void find_edges(Edges *e, const int32_t *cu, const int32_t *ckpt, int batch, int n_ckpt, int64_t T, int64_t t0, int threads)
{
    for (int b = threadIdx.x; b < batch; b += threads) {
        const RecSeq s = rec_seq(cu, b, T);
        const int64_t from = s.start - t0, to = s.start + (int64_t)s.n - 1 - t0;
        if (s.n > 0 && from >= 0 && from < kChunk)
            e->first[from] = b + 1;
        if (s.n > 0 && to >= 0 && to < kChunk)
            e->last[to] = b + 1;
    }
    for (int k = threadIdx.x; k < n_ckpt; k += threads) {
        const int64_t at = ckpt[k] - t0;
        if (at >= 0 && at < kChunk)
            e->ckpt[at] = 1;
    }
}
__device__ __forceinline__ void clear_edges(Edges *e)
{
    if (threadIdx.x < kChunk)
        e->first[threadIdx.x] = e->last[threadIdx.x] = e->ckpt[threadIdx.x] = 0;
}

// ---------------------------------------------------------------- the chunks in front
// The state in front of chunk `k` of a series of chunks (in the order in which they are taken) for this lane's channels; called by
// all waves of the workgroup.  wave w polls the maps w, w + W, ... of the chunk's group, the last wave also the state behind
// the group in front.
template <int V, int W> __device__ __forceinline__ void state_in_front(const Look &look, int k, int c, bool c_ok, float2 *lds_maps, float *lds_state, float *carry)
{
    const int l = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int group = k / kGroup, before = k - group * kGroup;
    constexpr int MOST = (kGroup - 1 + W - 1) / W;
    uint64_t map[MOST][V];
    uint32_t state[V];
    const bool wants_state = wave == W - 1 && group > 0;
    for (int polls = 0;; ++polls) {
        bool there = true;
#pragma unroll
        for (int u = 0; u < MOST; ++u) {
            const int j = wave + u * W;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                map[u][v] = 0;
                if (j < before && c_ok)
                    map[u][v] = load_published(look.maps + (int64_t)(group * kGroup + j) * look.channels + c + v);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            state[v] = 0;
            if (wants_state && c_ok)
                state[v] = load_published(look.states + (int64_t)(group - 1) * look.channels + c + v);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
            for (int u = 0; u < MOST; ++u)
                there = there && map[u][v] != ~0ull;
            there = there && state[v] != kNothing;
        }
        if (!__any(!there) || polls >= kMostPolls)
            break;
        __builtin_amdgcn_s_sleep(1);
    }
#pragma unroll
    for (int u = 0; u < MOST; ++u)
        if (wave + u * W < before)
#pragma unroll
            for (int v = 0; v < V; ++v)
                lds_maps[((wave + u * W) * 64 + l) * V + v] = make_float2(__uint_as_float((uint32_t)map[u][v]), __uint_as_float((uint32_t)(map[u][v] >> 32)));
    if (wave == W - 1)
#pragma unroll
        for (int v = 0; v < V; ++v)
            lds_state[l * V + v] = __uint_as_float(state[v]);
    lds_barrier();
#pragma unroll
    for (int v = 0; v < V; ++v)
        carry[v] = lds_state[l * V + v];
    for (int j = 0; j < before; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float2 m = lds_maps[(j * 64 + l) * V + v];
            carry[v] = apply(m.x, m.y, carry[v]);
        }
}
template <int V> __device__ __forceinline__ void publish_map(const Look &look, int k, int c, bool c_ok, const float *A, const float *H)
{
    if (c_ok)
#pragma unroll
        for (int v = 0; v < V; ++v)
            publish(look.maps + (int64_t)k * look.channels + c + v, (uint64_t)__float_as_uint(never_nothing(H[v])) << 32 | __float_as_uint(A[v]));
}
template <int V> __device__ __forceinline__ void publish_state(const Look &look, int k, int c, bool c_ok, const float *h)
{
    if (c_ok)
#pragma unroll
        for (int v = 0; v < V; ++v)
            publish(look.states + (int64_t)(k / kGroup) * look.channels + c + v, __float_as_uint(never_nothing(h[v])));
}

// ---------------------------------------------------------------- forward
template <int V, int W> struct ScanLds {
    Edges edges;
    float2 waves[W][64 * V];
    float2 maps[(kGroup - 1) * 64 * V];
    float state[64 * V];
    int taken;
};

template <typename E, int V, int W> __global__ __launch_bounds__(64 * W, 4) void rec_scan_kernel(RecScan a, Look look)
{
    constexpr int S = kChunk / W;
    static_assert(S % REC_SAVED_EVERY == 0, "saved states lie at the same tokens in all waves");
    extern __shared__ __align__(16) unsigned char lds_raw[];
    ScanLds<V, W> &lds = *reinterpret_cast<ScanLds<V, W> *>(lds_raw);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = tid & 63;
    const int C = look.channels, block = blockIdx.x % look.n_blocks;
    if (tid == 0)
        lds.taken = look.n_chunks > 1 ? __hip_atomic_fetch_add(look.tickets + block, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    clear_edges(&lds.edges);
    lds_barrier();
    const int chunk = __builtin_amdgcn_readfirstlane(lds.taken);
    const int64_t t0 = (int64_t)chunk * kChunk, first = t0 + wave * S;
    const int own = block * 64 * V + l * V;
    const bool c_ok = own < C;
    const int c = c_ok ? own : 0;

    typedef RecRow<E, V> Row;
    typename Row::Raw x[S], r[S], i[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t t = first + s < a.T ? first + s : a.T - 1;
        x[s] = row_load<E, V>(a.in.x, t, a.in.x_stride, c);
        r[s] = row_load<E, V>(a.in.r, t, a.in.r_stride, c);
        i[s] = row_load<E, V>(a.in.i, t, a.in.i_stride, c);
    }
    float rate[V];
    state_row_load<V>(look.rate, 0, C, c, rate);
    find_edges(&lds.edges, a.cu, a.ckpt, a.batch, a.n_ckpt, a.T, t0, 64 * W);
    const int cu0 = a.cu[0], cu1 = a.cu[a.batch];
    lds_barrier();
    // this wave's edges, as bits of its tokens
    const bool mine = l < S;
    const uint32_t firsts = (uint32_t)__ballot(mine && lds.edges.first[wave * S + (mine ? l : 0)] != 0);
    const uint32_t lasts = (uint32_t)__ballot(mine && lds.edges.last[wave * S + (mine ? l : 0)] != 0);
    const uint32_t wanted = (uint32_t)__ballot(mine && lds.edges.ckpt[wave * S + (mine ? l : 0)] != 0);
    const uint32_t inside = (uint32_t)__ballot(mine && first + l < a.T && first + l >= cu0 && first + l < cu1);
    const int whole = firsts == 0 ? S : __builtin_ctz(firsts);  // tokens in front of the first start take the state in front

    float h[S][V], P[S][V];  // as if the state in front were zero, and what is kept of it
    float A[V], H[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        A[v] = 1.f, H[v] = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (firsts >> s & 1) {
            const int b = __builtin_amdgcn_readfirstlane(lds.edges.first[wave * S + s]) - 1;
#pragma unroll
            for (int v = 0; v < V; ++v)
                H[v] = 0.f;
            if (a.init)
                state_row_load<V>(a.init, b, C, c, H);
        }
        float xv[V], rv[V], iv[V];
        Row::unpack(x[s], xv);
        Row::unpack(r[s], rv);
        Row::unpack(i[s], iv);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates_of(rv[v], iv[v], rate[v]);
            H[v] = __builtin_fmaf(g.a, H[v], added(g, xv[v]));
            A[v] *= g.a;
            h[s][v] = H[v], P[s][v] = A[v];
        }
    }
    float carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        A[v] = firsts != 0 ? kCut : A[v];
        carry[v] = 0.f;
        lds.waves[wave][l * V + v] = make_float2(A[v], H[v]);
    }
    lds_barrier();
    if (look.n_chunks > 1) {
        float all_A[V], all_H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            all_A[v] = 1.f, all_H[v] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 m = lds.waves[w][l * V + v];
                all_H[v] = apply(m.x, m.y, all_H[v]);
                all_A[v] = m.x < 0.f || all_A[v] < 0.f ? kCut : all_A[v] * m.x;
            }
        }
        const bool ends_group = chunk % kGroup == kGroup - 1;
        if (wave == 0 && !ends_group)
            publish_map<V>(look, chunk, c, c_ok, all_A, all_H);
        if (chunk > 0)
            state_in_front<V, W>(look, chunk, c, c_ok, lds.maps, lds.state, carry);
        if (wave == 0 && ends_group) {
            float behind[V];
#pragma unroll
            for (int v = 0; v < V; ++v)
                behind[v] = apply(all_A[v], all_H[v], carry[v]);
            publish_state<V>(look, chunk, c, c_ok, behind);
        }
    }
#pragma unroll
    for (int w = 0; w < W - 1; ++w)
        if (w < wave)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 m = lds.waves[w][l * V + v];
                carry[v] = apply(m.x, m.y, carry[v]);
            }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s % REC_SAVED_EVERY == 0 && a.saved && first + s < a.T && c_ok)
            state_row_store<V>(a.saved, (first + s) / REC_SAVED_EVERY, C, own, s == 0 ? carry : h[s ? s - 1 : 0]);
        if (s < whole)
#pragma unroll
            for (int v = 0; v < V; ++v)
                h[s][v] = __builtin_fmaf(P[s][v], carry[v], h[s][v]);
        if ((inside >> s & 1) != 0) {
            if (a.y && c_ok)
                row_store<E, V>(a.y, first + s, a.y_stride, own, h[s]);
            if ((lasts >> s & 1) != 0 && a.final_states) {
                const int b = __builtin_amdgcn_readfirstlane(lds.edges.last[wave * S + s]) - 1;
                if (c_ok)
                    state_row_store<V>(a.final_states, b, C, own, h[s]);
            }
            if ((wanted >> s & 1) != 0 && c_ok)
                for (int k = 0; k < a.n_ckpt; ++k)
                    if (a.ckpt[k] == first + s)
                        state_row_store<V>(a.ckpt_states, k, C, own, h[s]);
        }
    }
    if (chunk == 0) {  // what no token writes
        float none[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            none[v] = 0.f;
        if (a.final_states)
            for (int b0 = 64 * wave; b0 < a.batch; b0 += 64 * W) {
                uint64_t left = __ballot(b0 + l < a.batch && rec_seq(a.cu, b0 + l < a.batch ? b0 + l : 0, a.T).n == 0);
                for (; left != 0; left &= left - 1) {
                    const int b = b0 + __builtin_ctzll(left);
                    float s[V];
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        s[v] = 0.f;
                    if (a.init)
                        state_row_load<V>(a.init, b, C, c, s);
                    if (c_ok)
                        state_row_store<V>(a.final_states, b, C, own, s);
                }
            }
        for (int k0 = 64 * wave; k0 < a.n_ckpt; k0 += 64 * W) {
            const int t = k0 + l < a.n_ckpt ? a.ckpt[k0 + l] : 0;
            uint64_t left = __ballot(k0 + l < a.n_ckpt && (t < 0 || t < cu0 || t >= cu1 || t >= a.T));
            for (; left != 0; left &= left - 1)
                if (c_ok)
                    state_row_store<V>(a.ckpt_states, k0 + __builtin_ctzll(left), C, own, none);
        }
    }
}

// ---------------------------------------------------------------- backward
template <int V, int W> struct GradsLds {
    Edges edges;
    float2 waves[W][64 * V];
    float2 maps[(kGroup - 1) * 64 * V];
    float state[64 * V];
    int taken;
};

// `part` [chunks][channels]: every chunk's sum of the decay's gradients.
template <typename E, int V, int W> __global__ __launch_bounds__(64 * W, 4) void rec_grads_kernel(RecGrads a, Look look, float *part)
{
    constexpr int S = kChunk / W;
    static_assert(S == REC_SAVED_EVERY, "a wave begins with a saved state");
    extern __shared__ __align__(16) unsigned char lds_raw[];
    GradsLds<V, W> &lds = *reinterpret_cast<GradsLds<V, W> *>(lds_raw);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = tid & 63;
    const int C = look.channels, block = blockIdx.x % look.n_blocks;
    if (tid == 0)
        lds.taken = look.n_chunks > 1 ? __hip_atomic_fetch_add(look.tickets + block, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    clear_edges(&lds.edges);
    lds_barrier();
    const int order = __builtin_amdgcn_readfirstlane(lds.taken), chunk = look.n_chunks - 1 - order;
    const int64_t t0 = (int64_t)chunk * kChunk, first = t0 + wave * S;
    const int own = block * 64 * V + l * V;
    const bool c_ok = own < C;
    const int c = c_ok ? own : 0;

    typedef RecRow<E, V> Row;
    typename Row::Raw x[S], r[S], i[S], dy[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        const int64_t t = first + s < a.T ? first + s : a.T - 1;
        x[s] = row_load<E, V>(a.in.x, t, a.in.x_stride, c);
        r[s] = row_load<E, V>(a.in.r, t, a.in.r_stride, c);
        i[s] = row_load<E, V>(a.in.i, t, a.in.i_stride, c);
        dy[s] = typename Row::Raw();
        if (a.dy)
            dy[s] = row_load<E, V>(a.dy, t, a.dy_stride, c);
    }
    float rate[V], H[V];
    state_row_load<V>(look.rate, 0, C, c, rate);
    state_row_load<V>(a.saved, (first < a.T ? first : 0) / REC_SAVED_EVERY, C, c, H);
    find_edges(&lds.edges, a.cu, nullptr, a.batch, 0, a.T, t0, 64 * W);
    const int cu0 = a.cu[0], cu1 = a.cu[a.batch];
    lds_barrier();
    const bool mine = l < S;
    const uint32_t firsts = (uint32_t)__ballot(mine && lds.edges.first[wave * S + (mine ? l : 0)] != 0);
    const uint32_t lasts = (uint32_t)__ballot(mine && lds.edges.last[wave * S + (mine ? l : 0)] != 0);
    const uint32_t inside = (uint32_t)__ballot(mine && first + l < a.T && first + l >= cu0 && first + l < cu1);

    float keep[S][V], before[S][V];  // a, and the state in front of each token
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (firsts >> s & 1) {
            const int b = __builtin_amdgcn_readfirstlane(lds.edges.first[wave * S + s]) - 1;
#pragma unroll
            for (int v = 0; v < V; ++v)
                H[v] = 0.f;
            if (a.init)
                state_row_load<V>(a.init, b, C, c, H);
        }
        float xv[V], rv[V], iv[V];
        Row::unpack(x[s], xv);
        Row::unpack(r[s], rv);
        Row::unpack(i[s], iv);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates_of(rv[v], iv[v], rate[v]);
            before[s][v] = H[v], keep[s][v] = g.a;
            H[v] = __builtin_fmaf(g.a, H[v], added(g, xv[v]));
        }
    }
    // q of a sequence's last token is that of its final state
    auto behind_last = [&](int s, float *q) __attribute__((always_inline)) {
        const int b = __builtin_amdgcn_readfirstlane(lds.edges.last[wave * S + s]) - 1;
#pragma unroll
        for (int v = 0; v < V; ++v)
            q[v] = 0.f;
        if (a.d_final)
            state_row_load<V>(a.d_final, b, C, c, q);
    };
    float A[V], Q[V], carry[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        A[v] = 1.f, Q[v] = 0.f, carry[v] = 0.f;
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        if (lasts >> s & 1)
            behind_last(s, Q);
        float d[V];
        Row::unpack(dy[s], d);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Q[v] = keep[s][v] * (d[v] + Q[v]);
            A[v] *= keep[s][v];
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        lds.waves[wave][l * V + v] = make_float2(lasts != 0 ? kCut : A[v], Q[v]);
    lds_barrier();
    if (look.n_chunks > 1) {
        float all_A[V], all_H[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            all_A[v] = 1.f, all_H[v] = 0.f;
#pragma unroll
            for (int w = W - 1; w >= 0; --w) {
                const float2 m = lds.waves[w][l * V + v];
                all_H[v] = apply(m.x, m.y, all_H[v]);
                all_A[v] = m.x < 0.f || all_A[v] < 0.f ? kCut : all_A[v] * m.x;
            }
        }
        const bool ends_group = order % kGroup == kGroup - 1;
        if (wave == 0 && !ends_group)
            publish_map<V>(look, order, c, c_ok, all_A, all_H);
        if (order > 0)
            state_in_front<V, W>(look, order, c, c_ok, lds.maps, lds.state, carry);
        if (wave == 0 && ends_group) {
            float behind[V];
#pragma unroll
            for (int v = 0; v < V; ++v)
                behind[v] = apply(all_A[v], all_H[v], carry[v]);
            publish_state<V>(look, order, c, c_ok, behind);
        }
    }
#pragma unroll
    for (int w = W - 1; w > 0; --w)
        if (w > wave)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float2 m = lds.waves[w][l * V + v];
                carry[v] = apply(m.x, m.y, carry[v]);
            }
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        sum[v] = 0.f;
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
        if (lasts >> s & 1)
            behind_last(s, carry);
        float xv[V], rv[V], iv[V], d[V], dx[V], dr[V], di[V];
        Row::unpack(x[s], xv);
        Row::unpack(r[s], rv);
        Row::unpack(i[s], iv);
        Row::unpack(dy[s], d);
        const bool is_inside = (inside >> s & 1) != 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gates g = gates_of(rv[v], iv[v], rate[v]);
            const float dh = d[v] + carry[v];
            const float over = g.kept2 > 0.f ? __builtin_amdgcn_rsqf(g.kept2) : 0.f, beta = g.kept2 * over;
            const float log_a = g.log2_a * 0.69314718055994531f;
            const float six = g.si * xv[v];
            dx[v] = dh * beta * g.si;
            di[v] = dh * beta * six * (1.f - g.si);
            const float d_log = dh * (g.a * before[s][v] - g.a * g.a * over * six);
            dr[v] = d_log * log_a * (1.f - g.sr);
            sum[v] += is_inside ? d_log * g.sr : 0.f;
            carry[v] = g.a * dh;
            if (!is_inside)
                dx[v] = dr[v] = di[v] = 0.f;
        }
        if (first + s < a.T && c_ok) {
            row_store<E, V>(a.dx, first + s, C, own, dx);
            row_store<E, V>(a.dr, first + s, C, own, dr);
            row_store<E, V>(a.di, first + s, C, own, di);
        }
        if ((firsts >> s & 1) != 0 && a.d_init) {
            const int b = __builtin_amdgcn_readfirstlane(lds.edges.first[wave * S + s]) - 1;
            if (c_ok)
                state_row_store<V>(a.d_init, b, C, own, carry);
        }
    }
    lds_barrier();  // the waves' maps have been read
#pragma unroll
    for (int v = 0; v < V; ++v)
        lds.waves[wave][l * V + v].x = sum[v];
    lds_barrier();
    if (wave == 0 && c_ok) {
        float all[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            all[v] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
                all[v] += lds.waves[w][l * V + v].x;
        }
        state_row_store<V>(part, chunk, C, own, all);
    }
    if (chunk == 0 && a.d_init)
        for (int b0 = 64 * wave; b0 < a.batch; b0 += 64 * W) {
            uint64_t left = __ballot(b0 + l < a.batch && rec_seq(a.cu, b0 + l < a.batch ? b0 + l : 0, a.T).n == 0);
            for (; left != 0; left &= left - 1) {
                const int b = b0 + __builtin_ctzll(left);
                float q[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    q[v] = 0.f;
                if (a.d_final)
                    state_row_load<V>(a.d_final, b, C, c, q);
                if (c_ok)
                    state_row_store<V>(a.d_init, b, C, own, q);
            }
        }
}

// d_decay = sum over the chunks of `part`, times d(log a)/d(decay) per unit of sigmoid(r).  64 channels and 16 slices of the chunks
// per workgroup, in 64 bits.
constexpr int kSumSlices = 16;
__global__ __launch_bounds__(64 * kSumSlices) void rec_sum_kernel(const float *part, int n_chunks, int channels, const float *decay, float sharpness, float *d_decay)
{
    extern __shared__ __align__(16) unsigned char lds_raw[];
    double *const lds = reinterpret_cast<double *>(lds_raw);  // [slices][64]
    const int l = threadIdx.x & 63, slice = threadIdx.x / 64, own = blockIdx.x * 64 + l, c = own < channels ? own : 0;
    double sum = 0.0;
#pragma unroll 8
    for (int k = slice; k < n_chunks; k += kSumSlices)
        sum += (double)part[(int64_t)k * channels + c];
    lds[slice * 64 + l] = sum;
    lds_barrier();
    if (slice != 0 || own >= channels)
        return;
    double all = 0.0;
#pragma unroll
    for (int s = 0; s < kSumSlices; ++s)
        all += lds[s * 64 + l];
    d_decay[own] = (float)(all * (double)-sharpness / (1.0 + (double)expf(-decay[own])));
}

// Gradients of a batch without tokens.
__global__ __launch_bounds__(kPrepareThreads) void rec_no_tokens_kernel(float *to, const float *from, int64_t n, int64_t stride)
{
    for (int64_t k = (int64_t)blockIdx.x * kPrepareThreads + threadIdx.x; k < n; k += stride)
        to[k] = from ? from[k] : 0.f;
}

// ---------------------------------------------------------------- launches
constexpr int kScanWaves = 4, kGradsWaves = 8;

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// The workspace: maps, states behind groups, tickets, rates; for the gradients the chunks' sums and, where it has to be computed
// again, what the forward pass saves.
struct Workspace {
    size_t maps, states, tickets, rate, part, saved, bytes;
    int64_t n_chunks, n_groups;
    Workspace(int channels, int64_t T, int grads)
    {
        n_chunks = (T + kChunk - 1) / kChunk;
        n_groups = (n_chunks + kGroup - 1) / kGroup;
        maps = 0;
        states = maps + (size_t)n_chunks * channels * 8;
        tickets = up256(states + (size_t)n_groups * channels * 4);
        rate = up256(tickets + (size_t)((channels + 63) / 64) * 4);
        part = up256(rate + (size_t)channels * 4);
        saved = up256(part + (grads ? (size_t)n_chunks * channels * 4 : 0));
        bytes = up256(saved + (grads == 2 ? (size_t)((T + REC_SAVED_EVERY - 1) / REC_SAVED_EVERY) * channels * 4 : 0));
    }
};

Look make_look(const rec_shape_t &s, const Workspace &w, unsigned char *at, int V)
{
    Look k;
    k.maps = reinterpret_cast<uint64_t *>(at + w.maps);
    k.states = reinterpret_cast<uint32_t *>(at + w.states);
    k.tickets = reinterpret_cast<int *>(at + w.tickets);
    k.rate = reinterpret_cast<float *>(at + w.rate);
    k.channels = s.channels;
    k.n_chunks = (int)w.n_chunks;
    k.n_blocks = (s.channels + 64 * V - 1) / (64 * V);
    return k;
}

unsigned some_blocks(int64_t n)
{
    const int64_t blocks = (n + kPrepareThreads - 1) / kPrepareThreads;
    return (unsigned)(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
}

hipError_t prepare(const rec_shape_t &s, const Workspace &w, const Look &look, const float *decay, hipStream_t stream)
{
    const int64_t words = w.n_chunks > 1 ? (int64_t)((w.states - w.maps) / 4 + (size_t)w.n_groups * s.channels) : 0;
    const unsigned blocks = some_blocks(words > s.channels ? words : s.channels);
    hipLaunchKernelGGL(rec_prepare_kernel, dim3(blocks), dim3(kPrepareThreads), 0, stream, reinterpret_cast<uint32_t *>(look.maps), words, look.tickets,
                       look.n_blocks, look.rate, decay, s.sharpness, s.channels, (int64_t)blocks * kPrepareThreads);
    return hipGetLastError();
}

bool pairs(const void *p, int64_t stride, int bytes) { return reinterpret_cast<uintptr_t>(p) % (2 * bytes) == 0 && stride % 2 == 0; }
// Two channels per lane: half of the loads, where rows allow it.
bool two_channels(const rec_shape_t &s, const RecIo &in)
{
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    return s.channels % 2 == 0 && pairs(in.x, in.x_stride, e) && pairs(in.r, in.r_stride, e) && pairs(in.i, in.i_stride, e);
}

template <typename E, int V> hipError_t scan(const rec_shape_t &s, const RecScan &a, const Workspace &w, unsigned char *at, hipStream_t stream)
{
    const Look look = make_look(s, w, at, V);
    hipError_t e = prepare(s, w, look, a.decay, stream);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((rec_scan_kernel<E, V, kScanWaves>), dim3((unsigned)(look.n_blocks * w.n_chunks)), dim3(64 * kScanWaves), sizeof(ScanLds<V, kScanWaves>), stream, a,
                       look);
    return hipGetLastError();
}
template <typename E, int V> hipError_t grads(const rec_shape_t &s, const RecGrads &a, const Workspace &w, unsigned char *at, hipStream_t stream)
{
    const Look look = make_look(s, w, at, V);
    float *const part = reinterpret_cast<float *>(at + w.part);
    hipError_t e = prepare(s, w, look, a.decay, stream);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((rec_grads_kernel<E, V, kGradsWaves>), dim3((unsigned)(look.n_blocks * w.n_chunks)), dim3(64 * kGradsWaves), sizeof(GradsLds<V, kGradsWaves>), stream,
                       a, look, part);
    e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(rec_sum_kernel, dim3((unsigned)((s.channels + 63) / 64)), dim3(64 * kSumSlices), 64 * kSumSlices * sizeof(double), stream, part, look.n_chunks,
                       s.channels, a.decay, s.sharpness, a.d_decay);
    return hipGetLastError();
}

hipError_t copy_states(float *to, const float *from, int64_t n, hipStream_t stream)
{
    if (!to || n == 0 || to == from)
        return hipSuccess;
    const unsigned blocks = some_blocks(n);
    hipLaunchKernelGGL(rec_no_tokens_kernel, dim3(blocks), dim3(kPrepareThreads), 0, stream, to, from, n, (int64_t)blocks * kPrepareThreads);
    return hipGetLastError();
}

}  // namespace

size_t rec_scan_workspace(const rec_shape_t &s, int batch, int64_t T, int grads)
{
    return T == 0 || batch == 0 ? 0 : Workspace(s.channels, T, grads).bytes;
}

hipError_t launch_rec_scan(const rec_shape_t &s, const RecScan &a, void *workspace, hipStream_t stream)
{
    if (a.T == 0) {
        const hipError_t e = copy_states(a.final_states, a.init, (int64_t)a.batch * s.channels, stream);
        return e != hipSuccess ? e : copy_states(a.ckpt_states, nullptr, (int64_t)a.n_ckpt * s.channels, stream);
    }
    const Workspace w(s.channels, a.T, 0);
    unsigned char *const at = static_cast<unsigned char *>(workspace);
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    const bool two = two_channels(s, a.in) && pairs(a.decay, 0, 4) && pairs(a.init, 0, 4) && (!a.y || pairs(a.y, a.y_stride, e)) && pairs(a.final_states, 0, 4) &&
                     pairs(a.ckpt_states, 0, 4) && pairs(a.saved, 0, 4);
    if (s.io_dtype == REC_DT_F32)
        return two ? scan<RecF32, 2>(s, a, w, at, stream) : scan<RecF32, 1>(s, a, w, at, stream);
    if (s.io_dtype == REC_DT_BF16)
        return two ? scan<RecBf16, 2>(s, a, w, at, stream) : scan<RecBf16, 1>(s, a, w, at, stream);
    return two ? scan<RecF16, 2>(s, a, w, at, stream) : scan<RecF16, 1>(s, a, w, at, stream);
}

hipError_t launch_rec_grads(const rec_shape_t &s, const RecGrads &given, void *workspace, hipStream_t stream)
{
    RecGrads a = given;
    if (a.T == 0) {
        const hipError_t e = copy_states(a.d_decay, nullptr, s.channels, stream);
        return e != hipSuccess ? e : copy_states(a.d_init, a.d_final, (int64_t)a.batch * s.channels, stream);
    }
    const Workspace w(s.channels, a.T, a.saved ? 1 : 2);
    unsigned char *const at = static_cast<unsigned char *>(workspace);
    if (!a.saved) {
        RecScan f = {};
        f.in = a.in, f.decay = a.decay, f.init = a.init, f.cu = a.cu, f.T = a.T, f.batch = a.batch;
        f.saved = reinterpret_cast<float *>(at + w.saved);
        a.saved = f.saved;
        const hipError_t e = launch_rec_scan(s, f, workspace, stream);
        if (e != hipSuccess)
            return e;
    }
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    const bool two = two_channels(s, a.in) && pairs(a.init, 0, 4) && (!a.dy || pairs(a.dy, a.dy_stride, e)) && pairs(a.saved, 0, 4) && pairs(a.d_final, 0, 4) &&
                     pairs(a.dx, 0, e) && pairs(a.dr, 0, e) && pairs(a.di, 0, e) && pairs(a.d_init, 0, 4);
    if (s.io_dtype == REC_DT_F32)
        return two ? grads<RecF32, 2>(s, a, w, at, stream) : grads<RecF32, 1>(s, a, w, at, stream);
    if (s.io_dtype == REC_DT_BF16)
        return two ? grads<RecBf16, 2>(s, a, w, at, stream) : grads<RecBf16, 1>(s, a, w, at, stream);
    return two ? grads<RecF16, 2>(s, a, w, at, stream) : grads<RecF16, 1>(s, a, w, at, stream);
}
