// The gated recurrence over packed sequences, and its backward pass.
//
// h_t = a_t h_(t-1) + b_t is the composition of maps h -> a h + b, which compose as (A, H) then (A', H') = (A A', A' H + H').  A
// workgroup of 8 waves has a chunk of tokens, 16 per wave (8 in the backward pass), and 64 V channels, V neighbouring ones per lane:
// with 16-bit types and V = 2 rows of 256 bytes.  A lane composes its tokens from registers, the workgroup its waves, and the state
// in front of a chunk comes from the workgroups in front of it while the chunk's values wait in registers, so that inputs are read
// once and gates, which cost as much as the reads, are computed once.  Backwards the same with q_t = a_t (dy_t + q_(t+1)), what
// a state's gradient hands to the one in front, over chunks in falling order.
//
// A workgroup takes the number of its chunk from a counter of its channels when it starts: what it waits for is in the hands
// of workgroups that run already, whatever order they are started in, so every wait ends.  A chunk publishes its (A, H) at once, the
// last chunk of a group of 8 that of the group, the last one of 8 groups the state behind them: the state in front of a chunk is the
// last such state, the maps of the groups behind it and those of the chunks of its own group, in this order, so that sums do not
// depend on timing.  What is published is one 64-bit word per channel, which holds a pattern that no result has until it is there:
// no other memory has to be ordered by it.
//
// Memory bounds long batches, and beside it the wait for the state in front, 30 to 50 us of the first: a prompt of 32768 tokens of 4096
// channels in bf16 265 us, 1.09 GB at 4.1 TB/s where copies reach 4.9, vector units busy 53 % of the time;  13877 tokens of 2560
// channels forwards 73 us, 3.8 TB/s, backwards 139 us, 0.55 GB at 3.9 TB/s, vector units 40 %; with two channels per lane the backward
// pass has more than its 128 registers hold, and 50 MB of what it writes, and as much of what it reads, is scratch memory.  (One level of published maps and chunks
// of 64 tokens: 293, 85 and 219 us.)  Short ones are latency: a launch that empties the words, a ticket, lengths, inputs, two
// or three waits for words, 11 us for 800 tokens of 256 channels.
#include <cmath>
#include <type_traits>

#include "rec_common.h"

#ifndef REC_FEW_WORKGROUPS  // tests with small batches choose others
#define REC_FEW_WORKGROUPS 128
#endif

namespace {

constexpr int kWaves = 8;
constexpr int kScanTokens = 16, kGradsTokens = 8;  // of a wave
static_assert(kScanTokens % REC_SAVED_EVERY == 0 && kGradsTokens == REC_SAVED_EVERY, "a wave of the backward pass begins with a saved state");
constexpr int kGroup = 8;           // chunks of a group, and groups between published states
constexpr uint64_t kNothing = ~0ull;
constexpr int kMostPolls = 1 << 22; // of a wait: seconds; its result is NaN then, and the grid still drains
constexpr float kCut = -1.f;        // A of a map that forgets what was in front: a sequence starts in it
// Smaller 1 - a^2 are 0 to the gradients, as they are to the forward pass: the instructions for roots take denormals as 0, and the
// reciprocal root of 0 is infinity, which times the gate's gradient, next to 0 as well, is anything.  What is dropped is at most
// 2^-63 of what it multiplies.
constexpr float kSmallestNormal = 0x1p-126f;

// H' of a map (A, H) of `carry`, and the map of both
__device__ __forceinline__ float apply(float2 m, float carry) { return m.x < 0.f ? m.y : __builtin_fmaf(m.x, carry, m.y); }
__device__ __forceinline__ float2 then(float2 first, float2 m) { return make_float2(m.x < 0.f || first.x < 0.f ? kCut : first.x * m.x, apply(m, first.y)); }

struct Look {
    uint64_t *maps;    // [chunks][channels] of the chunks
    uint64_t *groups;  // [groups][channels] of the groups
    uint64_t *states;  // [groups / kGroup][channels] behind every kGroup groups
    int *tickets;      // [blocks of channels]
    float *rate;       // [channels]
    int32_t channels, n_chunks, n_blocks;
};
__device__ __forceinline__ uint64_t load_published(const uint64_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void publish(uint64_t *p, float2 m)
{
    const float H = m.y != m.y ? __uint_as_float(0x7fc00000u) : m.y;  // never the pattern of nothing
    __hip_atomic_store(p, (uint64_t)__float_as_uint(H) << 32 | __float_as_uint(m.x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ int take(const Look &look, int block) { return __hip_atomic_fetch_add(look.tickets + block, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A wave has `TOKENS` tokens of a chunk, a lane V neighbouring channels of them.
template <int V, int TOKENS> struct Place {
    static constexpr int kChunk = kWaves * TOKENS, kChannels = 64 * V;  // of a workgroup
    int wave, l, column;  // column: the first of the lane's channels among the workgroup's
    __device__ __forceinline__ Place() : wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64)), l(threadIdx.x & 63), column(l * V) {}
};

// ---------------------------------------------------------------- in front of a scan
// Nothing is published yet, no chunk is taken; the channels' rates, whose softplus would cost a chunk as much as two of its tokens.
constexpr int kPrepareThreads = 256;
__global__ __launch_bounds__(kPrepareThreads) void rec_prepare_kernel(uint64_t *words, int64_t n_words, int *tickets, int n_tickets, float *rate, const float *decay,
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
template <int CHUNK> struct Edges {
    int first[CHUNK], last[CHUNK], ckpt[CHUNK];  // sequence + 1 that begins or ends with the token; whether its state is wanted
    int any;
    __device__ __forceinline__ void clear()
    {
        static_assert(CHUNK <= 64 * kWaves, "a thread per token");
        if ((int)threadIdx.x < CHUNK)
            first[threadIdx.x] = last[threadIdx.x] = ckpt[threadIdx.x] = 0;
        if (threadIdx.x == 0)
            any = 0;
    }
};
// A thread's first sequence and checkpoint, which are asked for in front of the number of the chunk and of the inputs: loads come back
// in their order, and a wait for these behind the inputs would be one for the inputs.
struct FirstEdges {
    RecSeq seq;
    int ckpt;
    __device__ __forceinline__ FirstEdges(const int32_t *cu, const int32_t *ckpt_, int batch, int n_ckpt, int64_t T)
    {
        seq.start = seq.n = 0, ckpt = -1;
        if ((int)threadIdx.x < batch)
            seq = rec_seq(cu, threadIdx.x, T);
        if ((int)threadIdx.x < n_ckpt)
            ckpt = ckpt_[threadIdx.x];
    }
};
template <int CHUNK>
__device__ __forceinline__ void find_edges(Edges<CHUNK> *e, const FirstEdges &f, const int32_t *cu, const int32_t *ckpt, int batch, int n_ckpt, int64_t T, int t0)
{
    auto sequence = [&](int b, const RecSeq &s) __attribute__((always_inline)) {
        const int from = s.start - t0, to = s.start + s.n - 1 - t0;
        if (s.n > 0 && from >= 0 && from < CHUNK)
            e->first[from] = b + 1, e->any = 1;
        if (s.n > 0 && to >= 0 && to < CHUNK)
            e->last[to] = b + 1, e->any = 1;
    };
    auto wanted = [&](int t) __attribute__((always_inline)) {
        const uint32_t at = (uint32_t)t - (uint32_t)t0;
        if (at < CHUNK)
            e->ckpt[at] = 1, e->any = 1;
    };
    sequence(threadIdx.x, f.seq);
    for (int b = threadIdx.x + 64 * kWaves; b < batch; b += 64 * kWaves)
        sequence(b, rec_seq(cu, b, T));
    wanted(f.ckpt);
    for (int k = threadIdx.x + 64 * kWaves; k < n_ckpt; k += 64 * kWaves)
        wanted(ckpt[k]);
}

// ---------------------------------------------------------------- the chunks in front
// What is in front of a chunk: the maps of its group, those of the groups, a state (as the H of a map).
template <int CHANNELS> struct Front {
    float2 rows[2 * (kGroup - 1) + 1][CHANNELS];
};
// The state in front of chunk `k` of a series of chunks, in the order in which they are taken, for this lane's channels, and what
// the chunk has to publish; called by all waves of the workgroup.  `m`: the chunk's map, which the last wave knows.
template <int V, int TOKENS> __device__ __forceinline__ void state_in_front(const Look &look, const Place<V, TOKENS> &p, int k, int c, bool c_ok, Front<Place<V, TOKENS>::kChannels> &lds, const float2 *m, float *carry)
{
    const int C = look.channels;
    const bool last_wave = p.wave == kWaves - 1;
    const int group = k / kGroup, before = k % kGroup, block = group / kGroup, groups_before = group % kGroup;
    const bool ends_group = before == kGroup - 1, ends_block = ends_group && groups_before == kGroup - 1;
    if (!ends_group && last_wave && c_ok)
#pragma unroll
        for (int v = 0; v < V; ++v)
            publish(look.maps + (int64_t)k * C + c + v, m[v]);
    if (k == 0)
        return;
    // row j of what is in front, or null
    auto source = [&](int j, bool maps, bool rest) __attribute__((always_inline)) -> const uint64_t * {
        if (j < kGroup - 1)
            return maps && j < before ? look.maps + ((int64_t)group * kGroup + j) * C : nullptr;
        if (j < 2 * (kGroup - 1))
            return rest && j - (kGroup - 1) < groups_before ? look.groups + ((int64_t)block * kGroup + j - (kGroup - 1)) * C : nullptr;
        return rest && block > 0 && j == 2 * (kGroup - 1) ? look.states + (int64_t)(block - 1) * C : nullptr;
    };
    constexpr int MOST = (2 * (kGroup - 1) + kWaves) / kWaves;  // rows of a wave
    auto wait = [&](bool maps, bool rest) __attribute__((always_inline)) {
        uint64_t row[MOST][V];
        for (int polls = 0;; ++polls) {
            bool there = true;
#pragma unroll
            for (int u = 0; u < MOST; ++u) {
                const uint64_t *const from = source(p.wave + u * kWaves, maps, rest);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    row[u][v] = from && c_ok ? load_published(from + c + v) : 0;
            }
#pragma unroll
            for (int u = 0; u < MOST; ++u)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    there = there && row[u][v] != kNothing;
            if (!__any(!there) || polls >= kMostPolls)
                break;
            __builtin_amdgcn_s_sleep(4);
        }
#pragma unroll
        for (int u = 0; u < MOST; ++u)
            if (source(p.wave + u * kWaves, maps, rest))
#pragma unroll
                for (int v = 0; v < V; ++v)
                    lds.rows[p.wave + u * kWaves][p.column + v] = make_float2(__uint_as_float((uint32_t)row[u][v]), __uint_as_float((uint32_t)(row[u][v] >> 32)));
        lds_barrier();
    };
    // the last chunk of a group does not wait for what is in front of the group until it has published the group
    wait(true, !ends_group);
    if (ends_group) {
        if (!ends_block && last_wave && c_ok)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float2 all = make_float2(1.f, 0.f);
                for (int j = 0; j < kGroup - 1; ++j)
                    all = then(all, lds.rows[j][p.column + v]);
                publish(look.groups + (int64_t)group * C + c + v, then(all, m[v]));
            }
        wait(false, true);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        carry[v] = block > 0 ? lds.rows[2 * (kGroup - 1)][p.column + v].y : 0.f;
        for (int j = 0; j < groups_before; ++j)
            carry[v] = apply(lds.rows[kGroup - 1 + j][p.column + v], carry[v]);
        for (int j = 0; j < before; ++j)
            carry[v] = apply(lds.rows[j][p.column + v], carry[v]);
        if (ends_block && last_wave && c_ok)
            publish(look.states + (int64_t)block * C + c + v, make_float2(0.f, apply(m[v], carry[v])));
    }
}

// ---------------------------------------------------------------- forward
template <int V> struct ScanLds {
    typedef Place<V, kScanTokens> P;
    Edges<P::kChunk> edges;
    float2 waves[kWaves][P::kChannels];
    Front<P::kChannels> front;
    int taken;
};

template <typename E, int V> __global__ __launch_bounds__(64 * kWaves, 4) void rec_scan_kernel(RecScan a, Look look)
{
    constexpr int S = kScanTokens;
    typedef Place<V, S> P;
    typedef RecRow<E, V> Row;
    extern __shared__ __align__(16) unsigned char lds_raw[];
    ScanLds<V> &lds = *reinterpret_cast<ScanLds<V> *>(lds_raw);
    const P p;
    const int C = look.channels, T = (int)a.T, block = blockIdx.x % look.n_blocks;
    const int own = block * P::kChannels + p.column;
    const bool c_ok = own < C;
    const int c = c_ok ? own : 0;
    if (threadIdx.x == 0)
        lds.taken = look.n_chunks > 1 ? take(look, block) : 0;
    lds.edges.clear();
    const FirstEdges first_edges(a.cu, a.ckpt, a.batch, a.n_ckpt, a.T);
    const int cu0 = a.cu[0], cu1 = a.cu[a.batch];
    float rate[V];
    state_row_load<V>(look.rate, 0, C, c, rate);
    lds_barrier();
    const int chunk = __builtin_amdgcn_readfirstlane(lds.taken), t0 = chunk * P::kChunk, first = t0 + p.wave * S;
    find_edges(&lds.edges, first_edges, a.cu, a.ckpt, a.batch, a.n_ckpt, a.T, t0);

    lds_barrier();
    // the same twice: chunks in the middle of a sequence have no branches between their tokens
    auto body = [&](auto edges) __attribute__((always_inline)) {
        constexpr bool EDGES = decltype(edges)::value;
        typename Row::Raw x[S], r[S], i[S];
        const int row0 = first < T ? first : T - 1, rows = T - row0 < S ? T - row0 : S;
        const WaveRows<E> x_rows(a.in.x, row0, a.in.x_stride, rows, C), r_rows(a.in.r, row0, a.in.r_stride, rows, C), i_rows(a.in.i, row0, a.in.i_stride, rows, C);
        if (!EDGES || rows == S) {
            const uint32_t x_at = x_rows.at(0, c), r_at = r_rows.at(0, c), i_at = i_rows.at(0, c);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                x_rows.get(x_at, s, x[s]);
                r_rows.get(r_at, s, r[s]);
                i_rows.get(i_at, s, i[s]);
            }
        } else {  // rows behind the last one are read from that
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int row = s < rows ? s : rows - 1;
                x_rows.get(x_rows.at(row, c), 0, x[s]);
                r_rows.get(r_rows.at(row, c), 0, r[s]);
                i_rows.get(i_rows.at(row, c), 0, i[s]);
            }
        }
        // the edges of the wave's tokens, as bits
        const int bit = p.l % S, of_wave = p.wave * S;
        constexpr uint32_t ALL = (1u << S) - 1;
        const uint32_t firsts = (uint32_t)__ballot(lds.edges.first[of_wave + bit] != 0) & ALL, lasts = (uint32_t)__ballot(lds.edges.last[of_wave + bit] != 0) & ALL;
        const uint32_t wanted = (uint32_t)__ballot(lds.edges.ckpt[of_wave + bit] != 0) & ALL;
        const uint32_t inside = (uint32_t)__ballot(first + bit < T && first + bit >= cu0 && first + bit < cu1) & ALL;
        const int whole = firsts == 0 ? S : __builtin_ctz(firsts);  // tokens in front of the first start take the state in front
        auto sequence = [&](const int *of, int s) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(of[of_wave + s]) - 1; };

        float h[S][V], kept[S][V];  // as if the state in front were zero, and what is kept of it
        float2 m[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            m[v] = make_float2(1.f, 0.f);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (EDGES && (firsts >> s & 1) != 0) {
                float H[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    H[v] = 0.f;
                if (a.init)
                    state_row_load<V>(a.init, sequence(lds.edges.first, s), C, c, H);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    m[v].y = H[v];
            }
            float xv[V], rv[V], iv[V];
            Row::unpack(x[s], xv);
            Row::unpack(r[s], rv);
            Row::unpack(i[s], iv);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gates g = gates_of(rv[v], iv[v], rate[v]);
                m[v] = make_float2(m[v].x * g.a, __builtin_fmaf(g.a, m[v].y, added(g, xv[v])));
                h[s][v] = m[v].y, kept[s][v] = m[v].x;
            }
            __builtin_amdgcn_sched_barrier(0);  // tokens are not mixed: the registers would not hold them
        }
        float carry[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            carry[v] = 0.f;
            m[v].x = EDGES && firsts != 0 ? kCut : m[v].x;
            lds.waves[p.wave][p.column + v] = m[v];
        }
        lds_barrier();
        if (look.n_chunks > 1) {
            if (p.wave == kWaves - 1)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    m[v] = make_float2(1.f, 0.f);
                    for (int g = 0; g < kWaves; ++g)
                        m[v] = then(m[v], lds.waves[g][p.column + v]);
                }
            state_in_front(look, p, chunk, c, c_ok, lds.front, m, carry);
        }
        for (int g = 0; g < p.wave; ++g)
#pragma unroll
            for (int v = 0; v < V; ++v)
                carry[v] = apply(lds.waves[g][p.column + v], carry[v]);
        const WaveRows<E> y_rows(a.y, row0, a.y_stride, rows, C);
        const uint32_t y_at = y_rows.at(0, c);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (s % REC_SAVED_EVERY == 0 && a.saved && (!EDGES || first + s < T) && c_ok)
                state_row_store<V>(a.saved, (first + s) / REC_SAVED_EVERY, C, own, s == 0 ? carry : h[s ? s - 1 : 0]);
            if (!EDGES || s < whole)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    h[s][v] = __builtin_fmaf(kept[s][v], carry[v], h[s][v]), pin(h[s][v]);
            if (a.y && c_ok && (!EDGES || (inside >> s & 1) != 0))
                y_rows.put(y_at, s, Row::pack(h[s]));
            if (EDGES && (lasts >> s & 1) != 0 && a.final_states) {
                const int b = sequence(lds.edges.last, s);
                if (c_ok)
                    state_row_store<V>(a.final_states, b, C, own, h[s]);
            }
            if (EDGES && (wanted & inside) >> s & 1 && c_ok)
                for (int k = 0; k < a.n_ckpt; ++k)
                    if (a.ckpt[k] == first + s)
                        state_row_store<V>(a.ckpt_states, k, C, own, h[s]);
        }
    };
    if (lds.edges.any == 0 && t0 >= cu0 && t0 + P::kChunk <= (cu1 < T ? cu1 : T))
        body(std::false_type());
    else
        body(std::true_type());
    if (chunk == 0) {  // what no token writes
        float none[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            none[v] = 0.f;
        if (a.final_states)
            for (int b = p.wave; b < a.batch; b += kWaves)
                if (rec_seq(a.cu, b, a.T).n == 0 && c_ok) {
                    float s[V];
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        s[v] = 0.f;
                    if (a.init)
                        state_row_load<V>(a.init, b, C, c, s);
                    state_row_store<V>(a.final_states, b, C, own, s);
                }
        for (int k = p.wave; k < a.n_ckpt; k += kWaves) {
            const int t = a.ckpt[k];
            if ((t < 0 || t < cu0 || t >= cu1 || t >= T) && c_ok)
                state_row_store<V>(a.ckpt_states, k, C, own, none);
        }
    }
}

// ---------------------------------------------------------------- backward
template <int V> struct GradsLds {
    typedef Place<V, kGradsTokens> P;
    Edges<P::kChunk> edges;
    float2 waves[kWaves][P::kChannels];
    Front<P::kChannels> front;
    // The state in front of each token, which would not fit the registers beside the gates: 32 KB with two channels per lane, that
    // only its own lane reads.
    float before[kGradsTokens][64 * kWaves * V];
    int taken;
};

// `part` [chunks][channels]: every chunk's sum of the decay's gradients.
template <typename E, int V> __global__ __launch_bounds__(64 * kWaves, 4) void rec_grads_kernel(RecGrads a, Look look, float *part)
{
    constexpr int S = kGradsTokens;
    typedef Place<V, S> P;
    typedef RecRow<E, V> Row;
    extern __shared__ __align__(16) unsigned char lds_raw[];
    GradsLds<V> &lds = *reinterpret_cast<GradsLds<V> *>(lds_raw);
    const P p;
    const int C = look.channels, T = (int)a.T, block = blockIdx.x % look.n_blocks;
    const int own = block * P::kChannels + p.column;
    const bool c_ok = own < C;
    const int c = c_ok ? own : 0;
    if (threadIdx.x == 0)
        lds.taken = look.n_chunks > 1 ? take(look, block) : 0;
    lds.edges.clear();
    const FirstEdges first_edges(a.cu, nullptr, a.batch, 0, a.T);
    const int cu0 = a.cu[0], cu1 = a.cu[a.batch];
    float rate[V], before0[V];
    state_row_load<V>(look.rate, 0, C, c, rate);
    lds_barrier();
    const int order = __builtin_amdgcn_readfirstlane(lds.taken), chunk = look.n_chunks - 1 - order;
    const int t0 = chunk * P::kChunk, first = t0 + p.wave * S;
    find_edges(&lds.edges, first_edges, a.cu, nullptr, a.batch, 0, a.T, t0);
    state_row_load<V>(a.saved, (first < T ? first : 0) / REC_SAVED_EVERY, C, c, before0);

    lds_barrier();
    auto body = [&](auto edges) __attribute__((always_inline)) {
        constexpr bool EDGES = decltype(edges)::value;
        typename Row::Raw x[S], r[S], i[S], dy[S];
        const int row0 = first < T ? first : T - 1, rows = T - row0 < S ? T - row0 : S;
        const WaveRows<E> x_rows(a.in.x, row0, a.in.x_stride, rows, C), r_rows(a.in.r, row0, a.in.r_stride, rows, C), i_rows(a.in.i, row0, a.in.i_stride, rows, C),
            dy_rows(a.dy, row0, a.dy_stride, rows, C);
        if (!EDGES || rows == S) {
            const uint32_t x_at = x_rows.at(0, c), r_at = r_rows.at(0, c), i_at = i_rows.at(0, c), dy_at = dy_rows.at(0, c);
#pragma unroll
            for (int s = 0; s < S; ++s) {
                x_rows.get(x_at, s, x[s]);
                r_rows.get(r_at, s, r[s]);
                i_rows.get(i_at, s, i[s]);
                dy[s] = typename Row::Raw();
                if (a.dy)
                    dy_rows.get(dy_at, s, dy[s]);
            }
        } else {  // rows behind the last one are read from that
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int row = s < rows ? s : rows - 1;
                x_rows.get(x_rows.at(row, c), 0, x[s]);
                r_rows.get(r_rows.at(row, c), 0, r[s]);
                i_rows.get(i_rows.at(row, c), 0, i[s]);
                dy[s] = typename Row::Raw();
                if (a.dy)
                    dy_rows.get(dy_rows.at(row, c), 0, dy[s]);
            }
        }
        const int bit = p.l % S, of_wave = p.wave * S;
        constexpr uint32_t ALL = (1u << S) - 1;
        const uint32_t firsts = (uint32_t)__ballot(lds.edges.first[of_wave + bit] != 0) & ALL, lasts = (uint32_t)__ballot(lds.edges.last[of_wave + bit] != 0) & ALL;
        const uint32_t inside = (uint32_t)__ballot(first + bit < T && first + bit >= cu0 && first + bit < cu1) & ALL;
        auto sequence = [&](const int *of, int s) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(of[of_wave + s]) - 1; };
        // q of a sequence's last token is that of its final state
        auto behind_last = [&](int s, float *q) __attribute__((always_inline)) {
            float d[V];
#pragma unroll
            for (int v = 0; v < V; ++v)
                d[v] = 0.f;
            if (a.d_final)
                state_row_load<V>(a.d_final, sequence(lds.edges.last, s), C, c, d);
#pragma unroll
            for (int v = 0; v < V; ++v)
                q[v] = d[v];
        };
        const int own_lane = threadIdx.x * V;

        Gates gates[S][V];
        float2 m[V];
        float carry[V], H[V], Q[V], A[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            H[v] = before0[v], A[v] = 1.f, Q[v] = 0.f, carry[v] = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (EDGES && (firsts >> s & 1) != 0) {
                float d[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    d[v] = 0.f;
                if (a.init)
                    state_row_load<V>(a.init, sequence(lds.edges.first, s), C, c, d);
#pragma unroll
                for (int v = 0; v < V; ++v)
                    H[v] = d[v];
            }
            float xv[V], rv[V], iv[V];
            Row::unpack(x[s], xv);
            Row::unpack(r[s], rv);
            Row::unpack(i[s], iv);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                gates[s][v] = gates_of(rv[v], iv[v], rate[v]);
                lds.before[s][own_lane + v] = H[v];
                H[v] = __builtin_fmaf(gates[s][v].a, H[v], added(gates[s][v], xv[v]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int s = S - 1; s >= 0; --s) {
            if (EDGES && (lasts >> s & 1) != 0)
                behind_last(s, Q);
            float d[V];
            Row::unpack(dy[s], d);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Q[v] = gates[s][v].a * (d[v] + Q[v]);
                A[v] *= gates[s][v].a;
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            m[v] = make_float2(EDGES && lasts != 0 ? kCut : A[v], Q[v]);
            lds.waves[p.wave][p.column + v] = m[v];
        }
        lds_barrier();
        if (look.n_chunks > 1) {
            if (p.wave == kWaves - 1)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    m[v] = make_float2(1.f, 0.f);
                    for (int g = kWaves - 1; g >= 0; --g)
                        m[v] = then(m[v], lds.waves[g][p.column + v]);
                }
            state_in_front(look, p, order, c, c_ok, lds.front, m, carry);
        }
        for (int g = kWaves - 1; g > p.wave; --g)
#pragma unroll
            for (int v = 0; v < V; ++v)
                carry[v] = apply(lds.waves[g][p.column + v], carry[v]);
        float sum[V];
#pragma unroll
        for (int v = 0; v < V; ++v)
            sum[v] = 0.f;
        const WaveRows<E> dx_rows(a.dx, row0, C, rows, C), dr_rows(a.dr, row0, C, rows, C), di_rows(a.di, row0, C, rows, C);
        const uint32_t to = dx_rows.at(0, c);
#pragma unroll
        for (int s = S - 1; s >= 0; --s) {
            if (EDGES && (lasts >> s & 1) != 0)
                behind_last(s, carry);
#pragma unroll
            for (int v = 0; v < V; ++v)
                pin(gates[s][v].a), pin(gates[s][v].sr), pin(gates[s][v].si), pin(gates[s][v].kept2);
            float xv[V], d[V], dx[V], dr[V], di[V];
            Row::unpack(x[s], xv);
            Row::unpack(dy[s], d);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Gates &g = gates[s][v];
                const float dh = d[v] + carry[v];
                const float over = g.kept2 >= kSmallestNormal ? __builtin_amdgcn_rsqf(g.kept2) : 0.f;
                const float back = g.a * dh, add = dh * (g.kept2 * over) * g.si;
                dx[v] = add;
                di[v] = add * xv[v] * (1.f - g.si);
                const float d_log = back * __builtin_fmaf(-(g.a * over * g.si), xv[v], lds.before[s][own_lane + v]);
                dr[v] = d_log * (rate[v] * 0.69314718055994531f * g.sr) * (1.f - g.sr);
                const bool outside = EDGES && (inside >> s & 1) == 0;
                if (outside)
                    dx[v] = dr[v] = di[v] = 0.f;
                pin(dx[v]), pin(dr[v]), pin(di[v]);
                sum[v] = __builtin_fmaf(outside ? 0.f : d_log, outside ? 0.f : g.sr, sum[v]);
                carry[v] = back;
            }
            __builtin_amdgcn_sched_barrier(0);
            if (c_ok && (!EDGES || first + s < T)) {
                dx_rows.put(to, s, Row::pack(dx));
                dr_rows.put(to, s, Row::pack(dr));
                di_rows.put(to, s, Row::pack(di));
            }
            if (EDGES && (firsts >> s & 1) != 0 && a.d_init) {
                const int b = sequence(lds.edges.first, s);
                if (c_ok)
                    state_row_store<V>(a.d_init, b, C, own, carry);
            }
        }
        lds_barrier();  // the waves' maps have been read
#pragma unroll
        for (int v = 0; v < V; ++v)
            lds.waves[p.wave][p.column + v].x = sum[v];
        lds_barrier();
        if (p.wave == 0 && c_ok) {
            float all[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                all[v] = 0.f;
                for (int g = 0; g < kWaves; ++g)
                    all[v] += lds.waves[g][p.column + v].x;
            }
            state_row_store<V>(part, chunk, C, own, all);
        }
    };
    if (lds.edges.any == 0 && t0 >= cu0 && t0 + P::kChunk <= (cu1 < T ? cu1 : T))
        body(std::false_type());
    else
        body(std::true_type());
    if (chunk == 0 && a.d_init)
        for (int b = p.wave; b < a.batch; b += kWaves)
            if (rec_seq(a.cu, b, a.T).n == 0 && c_ok) {
                float q[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    q[v] = 0.f;
                if (a.d_final)
                    state_row_load<V>(a.d_final, b, C, c, q);
                state_row_store<V>(a.d_init, b, C, own, q);
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
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// The workspace: maps, states behind groups, tickets, rates; for the gradients the chunks' sums and, where it has to be computed
// again, what the forward pass saves.
struct Workspace {
    size_t maps, groups, states, tickets, rate, part, saved, bytes;
    int64_t n_chunks, words;
    Workspace(int channels, int64_t T, int chunk, int grads)
    {
        n_chunks = (T + chunk - 1) / chunk;
        const int64_t n_groups = (n_chunks + kGroup - 1) / kGroup, n_states = (n_groups + kGroup - 1) / kGroup;
        words = (n_chunks + n_groups + n_states) * channels;
        maps = 0;
        groups = maps + (size_t)n_chunks * channels * 8;
        states = groups + (size_t)n_groups * channels * 8;
        tickets = up256(states + (size_t)n_states * channels * 8);
        rate = up256(tickets + (size_t)((channels + 63) / 64) * 4);
        part = up256(rate + (size_t)channels * 4);
        saved = up256(part + (grads ? (size_t)n_chunks * channels * 4 : 0));
        bytes = up256(saved + (grads == 2 ? (size_t)((T + REC_SAVED_EVERY - 1) / REC_SAVED_EVERY) * channels * 4 : 0));
    }
};

Look make_look(const rec_shape_t &s, const Workspace &w, unsigned char *at, int channels)
{
    Look k;
    k.maps = reinterpret_cast<uint64_t *>(at + w.maps);
    k.groups = reinterpret_cast<uint64_t *>(at + w.groups);
    k.states = reinterpret_cast<uint64_t *>(at + w.states);
    k.tickets = reinterpret_cast<int *>(at + w.tickets);
    k.rate = reinterpret_cast<float *>(at + w.rate);
    k.channels = s.channels;
    k.n_chunks = (int)w.n_chunks;
    k.n_blocks = (s.channels + channels - 1) / channels;
    return k;
}

unsigned some_blocks(int64_t n)
{
    const int64_t blocks = (n + kPrepareThreads - 1) / kPrepareThreads;
    return (unsigned)(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
}

hipError_t prepare(const rec_shape_t &s, const Workspace &w, const Look &look, const float *decay, hipStream_t stream)
{
    const int64_t words = w.n_chunks > 1 ? w.words : 0;
    const unsigned blocks = some_blocks(words > s.channels ? words : s.channels);
    hipLaunchKernelGGL(rec_prepare_kernel, dim3(blocks), dim3(kPrepareThreads), 0, stream, look.maps, words, look.tickets, look.n_blocks, look.rate, decay, s.sharpness,
                       s.channels, (int64_t)blocks * kPrepareThreads);
    return hipGetLastError();
}

bool pairs(const void *p, int64_t stride, int bytes) { return reinterpret_cast<uintptr_t>(p) % (2 * bytes) == 0 && stride % 2 == 0; }
int64_t workgroups(const rec_shape_t &s, int64_t T, bool two, int chunk) { return (s.channels + (two ? 127 : 63)) / (two ? 128 : 64) * ((T + chunk - 1) / chunk); }
// Two channels per lane, half of the loads, where rows allow it and more than REC_FEW_WORKGROUPS are left: with one there are twice as
// many, which 256 compute units can all run at once (us, one channel and two; bf16, 1000 channels, scan of 1600 tokens, 104 workgroups,
// 14.0 and 15.8, of 3200, 200, 19.6 and 17.8, of 32768 tokens of 4096 channels 293 and 264; gradients of 800 tokens, 104, 16.7 and
// 18.5, of 1600, 200, 23.0 and 22.1, of 12800 tokens of 2560 channels 170 and 151).
bool two_channels(const rec_shape_t &s, const RecIo &in, int64_t T, int chunk)
{
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    return s.channels % 2 == 0 && workgroups(s, T, true, chunk) > REC_FEW_WORKGROUPS && pairs(in.x, in.x_stride, e) && pairs(in.r, in.r_stride, e) && pairs(in.i, in.i_stride, e);
}
constexpr int kScanChunk = Place<1, kScanTokens>::kChunk, kGradsChunk = Place<1, kGradsTokens>::kChunk;
bool scan_two(const rec_shape_t &s, const RecScan &a)
{
    const int e = s.io_dtype == REC_DT_F32 ? 4 : 2;
    return two_channels(s, a.in, a.T, kScanChunk) && pairs(a.init, 0, 4) && (!a.y || pairs(a.y, a.y_stride, e)) && pairs(a.final_states, 0, 4) && pairs(a.ckpt_states, 0, 4) &&
           pairs(a.saved, 0, 4);
}
// fp32: rows of one channel per lane are 256 bytes already (12800 tokens of 2560 channels 209 us, two channels 232)
bool grads_two(const rec_shape_t &s, const RecGrads &a)
{
    return s.io_dtype != REC_DT_F32 && two_channels(s, a.in, a.T, kGradsChunk) && pairs(a.init, 0, 4) && (!a.dy || pairs(a.dy, a.dy_stride, 2)) && pairs(a.saved, 0, 4) &&
           pairs(a.d_final, 0, 4) && pairs(a.dx, 0, 2) && pairs(a.dr, 0, 2) && pairs(a.di, 0, 2) && pairs(a.d_init, 0, 4);
}
// The forward pass that computes again what the backward pass is not given.
RecScan again_of(const RecGrads &a)
{
    RecScan f = {};
    f.in = a.in, f.decay = a.decay, f.init = a.init, f.cu = a.cu, f.T = a.T, f.batch = a.batch;
    return f;
}
constexpr int64_t kMostWorkgroups = 0xffffffffll / (64 * kWaves);  // a launch numbers its threads in 32 bits

template <typename K> hipError_t lds_limit(K kernel, size_t lds)
{
    return lds > 65536 ? hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) : hipSuccess;
}

template <typename E, int V> hipError_t scan(const rec_shape_t &s, const RecScan &a, unsigned char *at, hipStream_t stream)
{
    const Workspace w(s.channels, a.T, Place<V, kScanTokens>::kChunk, 0);
    const Look look = make_look(s, w, at, Place<V, kScanTokens>::kChannels);
    hipError_t e = prepare(s, w, look, a.decay, stream);
    if (e == hipSuccess)
        e = lds_limit(rec_scan_kernel<E, V>, sizeof(ScanLds<V>));
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((rec_scan_kernel<E, V>), dim3((unsigned)(look.n_blocks * w.n_chunks)), dim3(64 * kWaves), sizeof(ScanLds<V>), stream, a, look);
    return hipGetLastError();
}
template <typename E, int V> hipError_t grads(const rec_shape_t &s, const RecGrads &a, const Workspace &w, unsigned char *at, hipStream_t stream)
{
    const Look look = make_look(s, w, at, Place<V, kGradsTokens>::kChannels);
    float *const part = reinterpret_cast<float *>(at + w.part);
    hipError_t e = prepare(s, w, look, a.decay, stream);
    if (e == hipSuccess)
        e = lds_limit(rec_grads_kernel<E, V>, sizeof(GradsLds<V>));
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL((rec_grads_kernel<E, V>), dim3((unsigned)(look.n_blocks * w.n_chunks)), dim3(64 * kWaves), sizeof(GradsLds<V>), stream, a, look, part);
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
    if (T == 0 || batch == 0)
        return 0;
    const size_t scan = Workspace(s.channels, T, kScanChunk, 0).bytes;
    const size_t all = grads ? Workspace(s.channels, T, kGradsChunk, grads).bytes : 0;
    return scan > all ? scan : all;
}

bool rec_fits(const rec_shape_t &s, int64_t T, int grads)
{
    return workgroups(s, T, s.channels % 2 == 0 && !(grads && s.io_dtype == REC_DT_F32), grads ? kGradsChunk : kScanChunk) <= kMostWorkgroups;
}
bool rec_fits(const rec_shape_t &s, const RecScan &a) { return workgroups(s, a.T, scan_two(s, a), kScanChunk) <= kMostWorkgroups; }
bool rec_fits(const rec_shape_t &s, const RecGrads &a)
{
    return workgroups(s, a.T, grads_two(s, a), kGradsChunk) <= kMostWorkgroups && (a.saved || rec_fits(s, again_of(a)));
}

hipError_t launch_rec_scan(const rec_shape_t &s, const RecScan &a, void *workspace, hipStream_t stream)
{
    if (a.T == 0) {
        const hipError_t e = copy_states(a.final_states, a.init, (int64_t)a.batch * s.channels, stream);
        return e != hipSuccess ? e : copy_states(a.ckpt_states, nullptr, (int64_t)a.n_ckpt * s.channels, stream);
    }
    unsigned char *const at = static_cast<unsigned char *>(workspace);
    const bool two = scan_two(s, a);
    if (s.io_dtype == REC_DT_F32)
        return two ? scan<RecF32, 2>(s, a, at, stream) : scan<RecF32, 1>(s, a, at, stream);
    if (s.io_dtype == REC_DT_BF16)
        return two ? scan<RecBf16, 2>(s, a, at, stream) : scan<RecBf16, 1>(s, a, at, stream);
    return two ? scan<RecF16, 2>(s, a, at, stream) : scan<RecF16, 1>(s, a, at, stream);
}

hipError_t launch_rec_grads(const rec_shape_t &s, const RecGrads &given, void *workspace, hipStream_t stream)
{
    RecGrads a = given;
    if (a.T == 0) {
        const hipError_t e = copy_states(a.d_decay, nullptr, s.channels, stream);
        return e != hipSuccess ? e : copy_states(a.d_init, a.d_final, (int64_t)a.batch * s.channels, stream);
    }
    unsigned char *const at = static_cast<unsigned char *>(workspace);
    const bool again = !a.saved;
    const bool two = grads_two(s, a);
    const Workspace w(s.channels, a.T, kGradsChunk, again ? 2 : 1);
    if (again) {
        // its maps lie in front of what it saves
        const size_t maps = Workspace(s.channels, a.T, kScanChunk, 0).bytes;
        RecScan f = again_of(a);
        f.saved = reinterpret_cast<float *>(at + (w.saved > maps ? w.saved : maps));
        a.saved = f.saved;
        const hipError_t e = launch_rec_scan(s, f, workspace, stream);
        if (e != hipSuccess)
            return e;
    }
    if (s.io_dtype == REC_DT_F32)
        return grads<RecF32, 1>(s, a, w, at, stream);
    if (s.io_dtype == REC_DT_BF16)
        return two ? grads<RecBf16, 2>(s, a, w, at, stream) : grads<RecBf16, 1>(s, a, w, at, stream);
    return two ? grads<RecF16, 2>(s, a, w, at, stream) : grads<RecF16, 1>(s, a, w, at, stream);
}
