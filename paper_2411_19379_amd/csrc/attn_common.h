// What the attention kernels share (gfx950 only): arguments, how the work of a batch is dealt to workgroups, which keys a
// query sees, the cache's rows.
#pragma once

#include "attn_tree.h"
#include "mfma_utils.h"

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr int kMaxBatch = 4096;
constexpr int kMostWindow = 0x7fffff00;  // differences of positions and windows stay within 32 bits

// ---------------------------------------------------------------- lanes and waves
__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }
__device__ __forceinline__ int read_from(int v, int lane) { return __builtin_amdgcn_ds_bpermute(lane << 2, v); }
__device__ __forceinline__ float read_from(float v, int lane)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(lane << 2, (int)__float_as_uint(v)));
}

// LDS is ordered, loads in flight stay in flight
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void lds_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Where a pointer into LDS points, as the copies below want it.
__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p;
}
// The copies below write M0.  In front of a copy and behind it this tells the compiler, so that nothing that it keeps there lives
// across one: a value in M0 that a use in front needs stays in front, and a use behind gets its own.
__device__ __forceinline__ void m0_is_lost()
{
#ifdef __HIP_DEVICE_COMPILE__
    __asm__ volatile("" ::: "m0", "memory");
#endif
}
// 16 bytes per lane from memory right into LDS: lane l's, `offset` bytes behind `from`, go to `to` + 16 l; `from` and `to` are
// the same for the whole wave.  They are there after the wave's next memory_wait(); the wave must wait before it ends.
__device__ __forceinline__ void copy16_to_lds(const void *from, uint32_t offset, uint32_t to)
{
    m0_is_lost();
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(from), "s"(to) : "memory");
    m0_is_lost();
}
// The same with an address per lane.
__device__ __forceinline__ void copy16_to_lds(const void *from, uint32_t to)
{
    m0_is_lost();
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
    m0_is_lost();
}
__device__ __forceinline__ void memory_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// The value, of which the compiler knows nothing: what rare branches compute from it stays in them instead of taking registers
// of the loops around them.
template <typename T> __device__ __forceinline__ T unknown(T v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// A pointer, the same in all lanes, in scalar registers of its own.  Arguments are loaded sixteen registers at a time, and kept,
// spilled and read back like that for the sake of one of them.
__device__ __forceinline__ const unsigned char *own_pointer(const void *p)
{
    const uint64_t u = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane(unknown((int)(uint32_t)u)), hi = (uint32_t)__builtin_amdgcn_readfirstlane(unknown((int)(u >> 32)));
    return (const unsigned char *)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ uint32_t sat_add(uint32_t a, uint32_t b) { return a + b < a ? 0xffffffffu : a + b; }

#define ATTN_DPP(v, ctrl, row_mask, bound) __builtin_amdgcn_update_dpp(0, (int)(v), (ctrl), (row_mask), 0xF, (bound))
// Inclusive prefix sums over the lanes of a wave with DPP row shifts and the two row broadcasts.
__device__ __forceinline__ int wave_scan(int v)
{
    v += ATTN_DPP(v, 0x111, 0xF, true);   // row_shr:1
    v += ATTN_DPP(v, 0x112, 0xF, true);   // row_shr:2
    v += ATTN_DPP(v, 0x114, 0xF, true);   // row_shr:4
    v += ATTN_DPP(v, 0x118, 0xF, true);   // row_shr:8
    v += ATTN_DPP(v, 0x142, 0xA, false);  // row_bcast:15 into rows 1 and 3
    v += ATTN_DPP(v, 0x143, 0xC, false);  // row_bcast:31 into rows 2 and 3
    return v;
}
// The sum over the lanes, 2^32 - 1 if it does not fit: saturating sums do not depend on their order.
__device__ __forceinline__ uint32_t wave_sat_sum(uint32_t v)
{
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x111, 0xF, true));
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x112, 0xF, true));
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x114, 0xF, true));
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x118, 0xF, true));
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x142, 0xA, false));
    v = sat_add(v, (uint32_t)ATTN_DPP(v, 0x143, 0xC, false));
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// ---------------------------------------------------------------- arguments of attn_attend
struct AttendArgs {
    const void *q, *k_cache, *v_cache;
    const int32_t *table, *cu, *cached;
    void *out;
    float *lse;
    float *part;            // partial results: [part][rows_cap][D] sums, then [part][rows_cap][2] maximum and weight
    int64_t q_stride, out_stride;
    int64_t T;
    int32_t batch, Hq, Hkv, group;
    int32_t log2_bs, max_blocks, n_blocks;
    int32_t window, sinks;
    float scale_log2;       // scale * log2(e): the softmax runs on powers of two
    float outgrown;         // by how much a score may exceed a row's maximum before the row is scaled down
    int32_t rows_cap;       // rows of a partial result
    int32_t most_parts;     // partial results there is room for
    uint32_t target;        // workgroups that keep the GPU busy
    int32_t min_steps;      // a workgroup gets no fewer steps of keys than this if it can help it
    int32_t half_steps;     // up to so many it gets what it would get if half of the workgroups shared them
    // trees of new tokens; words is 0 where a sequence's new tokens follow one another
    const int32_t *positions, *seen;  // [T], [T, words]: bit j of row i: the query of new token i sees new token j
    int32_t words;
};

// ---------------------------------------------------------------- sequences
struct Seq {
    int start;   // first packed token
    int n;       // new tokens
    int cached;
    int rows;    // n * group: the row of token i and the group's head h is i * group + h
};
__device__ __forceinline__ Seq make_seq(const AttendArgs &a, int cu0, int cu1, int cached)
{
    Seq s;
    const int most = (int)a.T, from = cu0 < 0 ? 0 : cu0, to = cu1 > most ? most : cu1;
    s.start = from;
    s.n = to > from ? to - from : 0;
    s.cached = cached < 0 ? 0 : cached > 0x3fffffff ? 0x3fffffff : cached;
    s.rows = s.n * a.group;
    return s;
}
__device__ __forceinline__ Seq load_seq(const AttendArgs &a, int b) { return make_seq(a, a.cu[b], a.cu[b + 1], a.cached[b]); }

// Keys behind the end of the table's rows do not exist.
__device__ __forceinline__ int table_end(const AttendArgs &a)
{
    const int64_t keys = (int64_t)a.max_blocks << a.log2_bs;
    return keys > 0x7fffffff ? 0x7fffffff : (int)keys;
}

// Keys that the rows [r0, r0 + ROWS) of a sequence see, in tiles of KT keys: first the sinks' tiles, then those from `near` on.
struct KeyRange {
    int pos0, pos1;  // positions of the first and the last row
    int end;         // no row sees this key or one behind it
    int near;        // first tile of the window
    int n_sink;      // tiles of sinks in front of it
    int n;           // tiles in all
    __device__ __forceinline__ int tile(int step) const { return step < n_sink ? step : near + step - n_sink; }
};
template <int KT, bool TREE = false> __device__ __forceinline__ KeyRange key_range(const AttendArgs &a, const Seq &s, int r0, int rows)
{
    KeyRange k;
    const int last = r0 + rows < s.rows ? r0 + rows - 1 : s.rows - 1;
    // a tree's tokens lie one behind the other in the cache, and any of them may be the first behind the cached ones by its position
    k.pos0 = TREE ? s.cached : s.cached + r0 / a.group;
    k.pos1 = s.cached + last / a.group;
    const int most = table_end(a);
    k.end = k.pos1 < most ? k.pos1 + 1 : most;
    const int tiles = (k.end - 1) / KT + 1;
    const int lo = a.window > 0 && k.pos0 >= a.window ? k.pos0 - a.window + 1 : 0;
    k.near = lo / KT < tiles ? lo / KT : tiles;
    const int sink_tiles = a.sinks / KT + (a.sinks % KT != 0);
    k.n_sink = sink_tiles < k.near ? sink_tiles : k.near;
    k.n = k.n_sink + tiles - k.near;
    return k;
}
// How many steps the splits of a sequence are made for: those of its longest tile of rows, but for keys that the table has no
// place for, and no more than a window has.  The host computes the same bounds for any sequence (may_split).
template <int KT> __device__ __forceinline__ int window_steps(const AttendArgs &a, int rows)
{
    const int64_t near = ((int64_t)a.window + (a.words > 0 ? 32 * a.words : rows / a.group) + 1) / KT + 2 + ((int64_t)a.sinks + KT - 1) / KT;
    return a.window > 0 && near < 0x7fffffff ? (int)near : 0x7fffffff;
}

__device__ __forceinline__ bool sees(const AttendArgs &a, int pos, int j)
{
    return j <= pos && (a.window <= 0 || pos - j < a.window || j < a.sinks);
}
// Which of the N <= 64 keys from j0 on the query at `pos` sees, of those that exist: bit k is key j0 + k.
__device__ __forceinline__ uint64_t first_bits(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t seen_keys(const AttendArgs &a, int pos, int j0, uint64_t exist)
{
    uint64_t m = exist & first_bits(pos - j0 + 1);
    if (a.window > 0)
        m &= ~first_bits(pos - j0 - a.window + 1) | first_bits(a.sinks - j0);
    return m;
}
// Of a tree's token the query sees cached keys by its position, which lies between the first new one and the one that it would
// have in a chain, and new ones by its bits, up to its own.
__device__ __forceinline__ int tree_position(const AttendArgs &a, const Seq &s, int token)
{
    const int p = a.positions[s.start + token], most = s.cached + token;
    return p < s.cached ? s.cached : p > most ? most : p;
}
// The bits of new tokens [first, first + 64); `first` may be negative.
__device__ __forceinline__ uint64_t tree_bits(const AttendArgs &a, const Seq &s, int token, int first)
{
    const int32_t *const row = a.seen + (int64_t)(s.start + token) * a.words;
    const int w = first >> 5, shift = first & 31;
    uint32_t word[3];
#pragma unroll
    for (int k = 0; k < 3; ++k)
        word[k] = (uint32_t)(w + k) < (uint32_t)a.words ? (uint32_t)row[w + k] : 0u;
    const uint64_t low = (uint64_t)word[1] << 32 | word[0];
    const uint64_t bits = shift == 0 ? low : low >> shift | (uint64_t)word[2] << (64 - shift);
    return bits & first_bits(token - first + 1);
}
template <bool TREE> __device__ __forceinline__ uint64_t seen_keys(const AttendArgs &a, const Seq &s, int pos, int token, int j0, uint64_t exist)
{
    if (!TREE)
        return seen_keys(a, pos, j0, exist);
    const uint64_t cached = seen_keys(a, pos, j0, first_bits(s.cached - j0));
    return exist & (s.cached - j0 < 64 ? cached | tree_bits(a, s, token, j0 - s.cached) : cached);
}
template <bool TREE> __device__ __forceinline__ bool sees(const AttendArgs &a, const Seq &s, int pos, int token, int j)
{
    return TREE && j >= s.cached ? (tree_bits(a, s, token, j - s.cached) & 1) != 0 : sees(a, pos, j);
}
// The score, or minus infinity (a weight of 0 in any case) if `bit` of the keys that are seen is not set: two bit operations and
// no condition register.
__device__ __forceinline__ float seen_score(float score, uint32_t keys, int bit)
{
    const uint32_t is = (uint32_t)((int)(keys << (31 - bit)) >> 31);
    return __uint_as_float((__float_as_uint(score) & is) | (0xff800000u & ~is));
}

// Of which tiles of n keys every row at positions pos0..pos1 sees every key.  (Of a tree's rows every one sees the cached keys and,
// for all that is known here, no other: pos0 is the last cached position.)
struct SeenTiles {
    int last, behind, sinks;  // first keys: up to `last` and behind `behind`, or up to `sinks`
    __device__ __forceinline__ SeenTiles(const AttendArgs &a, int pos0, int pos1, int n)
        : last(pos0 - n + 1), behind(a.window > 0 ? pos1 - a.window : -1), sinks(a.sinks - n)
    {
    }
    __device__ __forceinline__ bool all(int j0) const { return j0 <= last && (j0 > behind || j0 <= sinks); }
};

// ---------------------------------------------------------------- who does what
// The rows of a sequence are cut into tiles of ROWS rows.  With `per` the steps of a workgroup if the GPU's `target` workgroups
// shared all steps, the tiles at a sequence's front that take no more than `per` stay whole, and the keys of all others are cut
// into the same number of splits, of about `per` steps if the tile is the last.  (2 requests of 100 and 300 tokens over 1000 to
// 4000 keys 41 us, with the number of splits rounded up 53; a prompt of 2000 tokens 110 us with every tile of it cut, 60 with the
// long ones.)  Every workgroup finds its own piece from the lengths: nothing is planned ahead, so the lengths may change between
// replays of a graph.
struct Item {
    int seq, tile, split, n_splits;
    int part;  // partial result: split s of key head h of this tile is (part + s) * Hkv + h
};
// The `unit`-th (tile, split) of the launch, or with `of_join` the unit-th tile of the sequences that are split; false if there is
// none.  Every wave finds out for itself, PER sequences per lane at a time: no barrier, one trip to memory for up to 64 PER
// sequences.  (With a sequence per thread, sums through LDS and its barriers it was 2.5 us of every workgroup's time.)
template <int PER, int ROWS, int KT> __device__ __forceinline__ bool find_among(const AttendArgs &a, int unit, bool of_join, Item *out)
{
    constexpr int ALL = 64 * PER;
    const int l = lane_id(), most_keys = table_end(a), most = window_steps<KT>(a, ROWS);
    int n[PER], cached[PER], tiles[PER], steps[PER];
    // no branch in it: all lengths are requested at once
    auto load = [&](int b0) __attribute__((always_inline)) {
        int from[PER + 1];
#pragma unroll
        for (int u = 0; u <= PER; ++u) {
            const int b = b0 + l * PER + u, at = b < a.batch ? b : a.batch;
            from[u] = a.cu[at];
            if (u < PER)
                cached[u] = a.cached[at < a.batch ? at : a.batch - 1];
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const Seq s = make_seq(a, from[u], from[u + 1], cached[u]);
            n[u] = s.n, cached[u] = s.cached;
            tiles[u] = (s.rows + ROWS - 1) / ROWS;
            const int keys = s.cached + s.n < most_keys ? s.cached + s.n : most_keys, all = (keys - 1) / KT + 1;
            steps[u] = s.n == 0 ? 0 : all < most ? all : most;
        }
    };
    uint32_t work = 0;  // steps of all workgroups
    for (int b0 = 0; b0 < a.batch; b0 += ALL) {
        load(b0);
        uint32_t w = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const uint64_t x = (uint64_t)tiles[u] * (uint64_t)steps[u] * (uint64_t)a.Hkv;
            w = sat_add(w, x > 0xffffffffu ? 0xffffffffu : (uint32_t)x);
        }
        work = sat_add(work, wave_sat_sum(w));
    }
    uint32_t per = work / a.target + (work % a.target != 0);  // steps of a workgroup
    if (a.half_steps > 0) {
        const uint32_t half = a.target / 2, twice = work / half + (work % half != 0), most = a.half_steps;
        const uint32_t least = twice < most ? twice : most;
        per = per < least ? least : per;
    }
    per = per < (uint32_t)a.min_steps ? (uint32_t)a.min_steps : per;
    per = work == 0xffffffffu ? 0x7fffffffu : per;  // a sum that did not fit says nothing but that there are tiles enough

    int items_before = 0, parts_before = 0;
    for (int b0 = 0; b0 < a.batch; b0 += ALL) {
        if (a.batch > ALL)
            load(b0);
        int splits[PER], whole[PER], items = 0, parts = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            splits[u] = (int)(((uint32_t)steps[u] + per / 2) / per);
            // of the first tiles, that take no more than `per` steps; with a window the steps hardly depend on the tile
            const int keys = (int)(((uint32_t)steps[u] < per ? (uint32_t)steps[u] : per) * KT - (uint32_t)cached[u]);
            const int short_tiles = a.window > 0 || keys <= 0 ? 0 : keys >= n[u] ? tiles[u] : keys * a.group / ROWS;
            whole[u] = splits[u] > 1 ? short_tiles : tiles[u];
            const int cut = tiles[u] - whole[u];
            items += of_join ? cut : whole[u] + cut * splits[u];
            parts += cut * splits[u];
        }
        const int items_upto = wave_scan(items), parts_upto = wave_scan(parts);
        int at = unit - items_before - (items_upto - items);
        const uint64_t here = __ballot(at >= 0 && at < items);
        if (here != 0) {
            int found = 0, n_splits = 1, n_whole = 0, left = 0, part = parts_before + parts_upto - parts;
            bool done = false;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int cut = tiles[u] - whole[u], n = of_join ? cut : whole[u] + cut * splits[u];
                if (!done && at < n) {
                    found = b0 + l * PER + u, n_splits = splits[u], n_whole = whole[u], left = n - 1 - at;  // the last rows, which see the most keys, first
                    done = true;
                }
                if (!done) {
                    at -= n;
                    part += cut * splits[u];
                }
            }
            const int owner = __builtin_ctzll(here);
            out->seq = __builtin_amdgcn_readlane(found, owner);
            n_splits = __builtin_amdgcn_readlane(n_splits, owner);
            n_whole = __builtin_amdgcn_readlane(n_whole, owner);
            left = __builtin_amdgcn_readlane(left, owner);
            part = __builtin_amdgcn_readlane(part, owner);
            if (!of_join && left < n_whole) {
                out->tile = left, out->split = 0, out->n_splits = 1, out->part = 0;
                return true;
            }
            const int of_cut = of_join ? left * n_splits : left - n_whole, tile = of_cut / n_splits;
            out->tile = n_whole + tile;
            out->split = of_cut - tile * n_splits;
            out->n_splits = n_splits;
            out->part = part + tile * n_splits;
            return true;
        }
        items_before += __builtin_amdgcn_readlane(items_upto, 63);
        parts_before += __builtin_amdgcn_readlane(parts_upto, 63);
    }
    return false;
}
// A sequence per lane as long as that reaches: 64 requests of one token 73 us, four per lane 77; 65 to 128 requests the same either
// way, 256 with four per lane 214, with one 218.
template <int ROWS, int KT> __device__ __forceinline__ bool find_item(const AttendArgs &a, int unit, bool of_join, Item *out)
{
    return a.batch <= 64 ? find_among<1, ROWS, KT>(a, unit, of_join, out) : find_among<4, ROWS, KT>(a, unit, of_join, out);
}
__device__ __forceinline__ int part_of(const AttendArgs &a, const Item &it, int kv_head, int split)
{
    return (it.part + split) * a.Hkv + kv_head;
}

// ---------------------------------------------------------------- the cache
// Row of the key at position j in a cache of [n_blocks * n_kv_heads * block_size] rows, or -1 if the table names no block
// for it.  The host has checked that rows fit 31 bits; byte offsets take 64.
__device__ __forceinline__ int cache_row(const AttendArgs &a, int block, int kv_head, int j)
{
    if ((uint32_t)block >= (uint32_t)a.n_blocks)
        return -1;
    return ((block * a.Hkv + kv_head) << a.log2_bs) + (j & ((1 << a.log2_bs) - 1));
}

// ---------------------------------------------------------------- 16-bit types
struct Bf16 {
    static constexpr uint32_t kExp = 0x7f80u;
    static constexpr float kPowers = 0.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack2_bf16(lo, hi); }
    static __device__ __forceinline__ float lo(uint32_t u) { return bf16_lo(u); }
    static __device__ __forceinline__ float hi(uint32_t u) { return bf16_hi(u); }
    static __device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c) { return mfma_bf16(a, b, c); }
    static __device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct F16 {
    static constexpr uint32_t kExp = 0x7c00u;
    static constexpr float kPowers = 7.f;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack2_f16(lo, hi); }
    static __device__ __forceinline__ float lo(uint32_t u) { return f16_lo(u); }
    static __device__ __forceinline__ float hi(uint32_t u) { return f16_hi(u); }
    static __device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c) { return mfma_f16(a, b, c); }
    static __device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

// Infinities and NaN of two packed values become zeros; true if there were any.
template <typename E> __device__ __forceinline__ bool drop_not_finite(uint32_t &u)
{
    const bool lo = (u & E::kExp) == E::kExp, hi = ((u >> 16) & E::kExp) == E::kExp;
    u = (lo ? 0u : u & 0xffffu) | (hi ? 0u : u & 0xffff0000u);
    return lo || hi;
}

// p v where v is not finite and the row sees its key (sees: all bits, or none), else 0, without a condition register.
__device__ __forceinline__ float not_finite_part(float p, float v, uint32_t sees)
{
    const uint32_t is = (uint32_t)((int)((__float_as_uint(v) & 0x7f800000u) + 0x00800000u) >> 31);
    return __uint_as_float(__float_as_uint(p * v) & is & sees);
}

// Weights are 2^(scale_log2 (score - m) + powers of the type).  The product with v takes them rounded to 16 bits, the sum of weights
// as they are.  In fp16 a weight below 2^-25 is nothing to the product, but counts in the sum: so the largest of a row is 2^7 (and
// 2^15 where m lags behind, which fp16 still holds), and keys count down to 2^-32 of it (behind a key of weight 1 and value 0, 1500
// of 2^-24 to 2^-28 came out as three quarters of their sum).
template <typename E> struct Weights {
    static constexpr float kPowers = E::kPowers;
};
template <> struct Weights<float> {
    static constexpr float kPowers = 0.f;
};
// What is subtracted from a row's scaled scores.  The maximum is taken as 0 where nothing finite has been seen yet, so that no
// infinity is subtracted from itself.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
template <typename E> __device__ __forceinline__ float subtrahend(float m, float scale_log2)
{
    constexpr float powers = Weights<E>::kPowers;
    return powers == 0.f ? finite_max(m) * scale_log2 : __builtin_fmaf(finite_max(m), scale_log2, -powers);
}

// How a row without any weight is marked in a partial result: it saw no key (0), or only scores of minus infinity or beyond fp32,
// of which the softmax is undefined (-1).
__device__ __forceinline__ float row_weight(float l, bool seen) { return l == 0.f && seen ? -1.f : l; }

// ln of the sum of exponentials of a row with this maximum and sum of weights.
template <typename E> __device__ __forceinline__ float row_lse(float m, float w, float scale_log2)
{
    if (w == 0.f)
        return -INFINITY;
    return w < 0.f ? NAN : (m * scale_log2 + (__builtin_amdgcn_logf(w) - Weights<E>::kPowers)) * 0.69314718055994531f;
}

// A row put together from partial results (maximum, weight): first every maximum, then every weight.
struct JoinedRow {
    float m = -INFINITY, w = 0.f;
    bool undefined = false;  // a part saw keys and has no weight
    __device__ __forceinline__ void add_max(float part_m) { m = fmaxf(m, part_m); }
    // the factor of the part's sums; 0 if the part has none
    __device__ __forceinline__ float add_weight(float part_m, float part_w, float scale_log2)
    {
        undefined = undefined || part_w < 0.f;
        if (part_w == 0.f || part_w < 0.f)
            return 0.f;
        // a part without a maximum and with weight has seen a NaN and nothing larger than minus infinity
        const float f = part_m == m ? 1.f : exp2_fast((finite_max(part_m) - m) * scale_log2);
        w += part_w * f;
        return f;
    }
    __device__ __forceinline__ float weight() const { return w == 0.f && undefined ? -1.f : w; }
    __device__ __forceinline__ float scale() const { return w == 0.f ? (undefined ? NAN : 0.f) : 1.f / w; }
};

}  // namespace

// Launchers implemented next to their kernels.
hipError_t launch_attn_assign(int batch, int log2_bs, int max_blocks, int64_t T, const int32_t *cu, const int32_t *cached,
                              const int32_t *shared, const int32_t *table_in, int32_t *table_out, const int32_t *free_blocks,
                              const int32_t *n_free, int32_t free_capacity, int64_t *slots, int32_t *positions, int32_t *copies,
                              int32_t *counts, hipStream_t stream);
hipError_t launch_attn_rope(const attn_shape_t &s, int64_t T, int batch, int n_blocks, const void *q, int64_t q_stride,
                            const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *positions,
                            const int64_t *slots, const float *rotary, int max_positions, int rotary_dim, bool interleaved,
                            const int32_t *copies, void *q_out, void *k_cache, void *v_cache, hipStream_t stream);
// The trees of a batch's new tokens; none (0 words): they follow one another.
struct AttnTrees {
    const int32_t *positions = nullptr, *seen = nullptr;
    int32_t words = 0;
};
hipError_t launch_attn_attend(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, const void *q,
                              int64_t q_stride, const void *k_cache, const void *v_cache, const int32_t *table,
                              const int32_t *cu, const int32_t *cached, float scale, int window, int sinks, int max_new,
                              void *out, int64_t out_stride, float *lse, void *workspace, hipStream_t stream,
                              const AttnTrees &trees = AttnTrees());
size_t attn_attend_tree_workspace(const attn_shape_t &s, int batch, int64_t T, int max_new);
hipError_t launch_attn_attend_tree(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, const void *q,
                                   int64_t q_stride, const void *k_cache, const void *v_cache, const int32_t *table,
                                   const int32_t *cu, const int32_t *cached, float scale, int window, int sinks, int max_new,
                                   void *out, int64_t out_stride, float *lse, void *workspace, hipStream_t stream, const AttnTrees &trees);
constexpr int kMostTreeWords = 32;   // a tree has up to 1024 tokens
constexpr int kCachesPerLaunch = 32; // their pointers travel in the kernel's arguments
hipError_t launch_attn_draft_tree(int batch, int64_t T, int words, const int32_t *parents, const int32_t *cu, const int32_t *cached,
                                  int window, int sinks, int32_t *positions, int32_t *seen, hipStream_t stream);
hipError_t launch_attn_accept(int batch, int log2_bs, int max_blocks, int64_t T, const int32_t *tokens, const int32_t *parents,
                              const int32_t *choices, const int32_t *cu, const int32_t *cached, const int32_t *table,
                              int32_t *free_blocks, const int32_t *n_free, int32_t free_capacity, int32_t *path, int32_t *counts,
                              int32_t *next_tokens, int32_t *kept_lens, int32_t *n_free_out, hipStream_t stream);
hipError_t launch_attn_keep(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, int n_caches,
                            void *const *caches, const int32_t *table, const int32_t *cu, const int32_t *cached,
                            const int32_t *path, hipStream_t stream);
size_t attn_attend_workspace(const attn_shape_t &s, int batch, int64_t T, int max_new);
