// Attention of the new tokens of a packed batch over the paged cache: for chunks of prompts, for single tokens, and in fp32.
//
// One pass over the keys with a running maximum m and weight l per row:  p = 2^(c (s - m)),  l = sum p,  O = sum p v,  with
// c = scale log2(e); when a row's scores outgrow m, what has been summed is scaled down.  With 16-bit types p is rounded to the type
// for the product with v, since the matrix instructions take no other, and l is the sum of what has not been rounded; all sums
// are fp32.  A query head reads the key head of its group, so the rows of a sequence are (token, head of the group) pairs: all
// that read one key head.
//
// All three kernels compute S^T = K Q^T, keys down the matrix rows, so that a lane holds scores of one row of the problem and
// keeps that row's m and l in registers, and O^T = V^T P^T, of which the lane's accumulators are the same row again.  The
// accumulators of S^T are, packed, already the operand P^T of the second product, with the keys in an order that the operand
// V^T is read in as well: P never leaves the registers.
//
// Rows that see only part of a tile of keys take their weights of the others as zero, and V's infinities and NaN in such
// tiles stay out of the matrix product (0 * inf is not 0): they are added to the rows that see them one key at a time.
#include <cfloat>

#include "attn_common.h"

#ifndef ATTN_TARGET  // workgroups that a launch is dealt to, where tests do not choose them
#define ATTN_TARGET 0
#endif

namespace {

constexpr float kOutgrown = 8.f;  // powers of two by which a weight may exceed that of the maximum before its row is scaled down

template <typename E> __device__ __forceinline__ void unpack4(uint2 u, float *v)
{
    v[0] = E::lo(u.x), v[1] = E::hi(u.x), v[2] = E::lo(u.y), v[3] = E::hi(u.y);
}

// ================================================================ chunks
// A workgroup takes 32 rows per wave and walks the keys in tiles of 64, K and V in LDS in three buffers each.
//
// A wave alternates between products, O += V^T(t-1) P^T(t-1) and S = K(t) Q^T, and the softmax of tile t on the vector ALUs;
// a tile costs about the same in both.  The two waves of a SIMD are kept one such phase apart by the workgroup's barriers, so
// that one's products run under the other's softmax: side by side in the same phase the two kinds of work took turns.
//
// With phases numbered from 0, the first half of the waves does products t in phase 2t and softmax t in phase 2t + 1, the other
// half one phase later.  V(t + 1) and K(t + 2) are requested at the start of a wave's softmax t, phase 2t + 1 or 2t + 2, behind
// the last reads of what they replace, V(t - 2) and K(t - 1) in phase 2t - 1; a wave waits for what it has requested at the end
// of its products t + 1, phase 2t + 2 or 2t + 3, and the first reads are in phase 2t + 4.
//
// With 128 values per head a tile of a wave is 1024 cycles of products and about 870 of softmax: the matrix cores bind, at the
// clock that the power allows (32768 tokens over 16384 cached, 32 heads, bf16: 15.1 ms, 1160 TFLOP/s, matrix cores busy 62 % of
// the cycles at 1.8 GHz; a library's product of 16384 reaches 1580).  With 64 the products are half as many and the softmax the
// same, which binds: 188 vector instructions per tile and wave, those around the loop included, beside 16 matrix instructions (16
// packed prompts of 512 to 4096 tokens, 16 heads, fp16: 312 us, 630 TFLOP/s).  There the pieces also go out sequence by sequence,
// which by their steps ends 27 % behind an even spread over the 512 workgroups that are resident, and 9 registers (14 with blocks of
// fewer than 8 tokens) go to memory at the 128 that four waves of a SIMD leave each other.  A tile of 256 rows by 64 keys needs
// 32 KB from the L2 for some 2 us.
constexpr int kChunkKeys = 64;

constexpr int kChunkBuffers = 3;

template <int D> struct ChunkTile {
    static constexpr int kPieces = D / 8;  // 16-byte pieces of a row
    static constexpr int kBytes = kChunkKeys * D * 2;
    // Piece c of row r lies at piece c ^ turn(r) of the row.  K is read 32 rows at a piece, V 8 rows at four neighbouring pieces:
    // both without two lanes of a group on one bank.
    static __device__ __forceinline__ int k_turn(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_turn(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
    static __device__ __forceinline__ int k_at(int r, int c) { return r * D * 2 + ((c ^ k_turn(r)) << 4); }
    static __device__ __forceinline__ int v_at(int r, int c) { return r * D * 2 + ((c ^ v_turn(r)) << 4); }
};

template <typename E, int D, int NW, bool WIDE> __global__ __launch_bounds__(64 * NW, D == 64 ? 4 : 2) void attn_chunk_kernel(AttendArgs a)
{
    typedef ChunkTile<D> Tile;
    constexpr int ROWS = 32 * NW, PIECES = Tile::kPieces;
    constexpr int KEYS = kChunkKeys / NW;        // of a tile, that a wave moves
    constexpr int LOADS = KEYS * PIECES / 64;    // copies of K (and of V) for them
    constexpr int ROWS_PER_LOAD = 64 / PIECES;
    static_assert(LOADS * ROWS_PER_LOAD == KEYS && KEYS == 8 && NW % 2 == 0, "whole tiles; KEYS is also the smallest wide block");
    extern __shared__ __align__(16) unsigned char lds_raw[];
    unsigned char *const lds_k = lds_raw, *const lds_v = lds_raw + kChunkBuffers * Tile::kBytes;
    // of four tiles: which keys exist, and whose V is not finite
    int *const lds_exist = reinterpret_cast<int *>(lds_raw + 2 * kChunkBuffers * Tile::kBytes), *const lds_bad = lds_exist + 4 * kChunkKeys;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = lane_id(), half = l / 32;
    const bool late = wave >= NW / 2;  // one phase behind the others
    const int kv_head = blockIdx.x % a.Hkv;
    Item it;
    if (!find_item<ROWS, kChunkKeys>(a, blockIdx.x / a.Hkv, false, &it))
        return;
    const Seq s = load_seq(a, it.seq);
    const int r0 = it.tile * ROWS;
    const KeyRange keys = key_range<kChunkKeys>(a, s, r0, ROWS);
    const int step_begin = (int)((int64_t)keys.n * it.split / it.n_splits);
    const int n = (int)((int64_t)keys.n * (it.split + 1) / it.n_splits) - step_begin;
    const int end = keys.end;

    // this lane's row
    const int row = r0 + 32 * wave + l % 32;
    const bool wave_works = r0 + 32 * wave < s.rows, row_works = row < s.rows;
    const int token = row_works ? row / a.group : 0, head = kv_head * a.group + (row_works ? row - token * a.group : 0);
    const int pos = s.cached + token;
    const int wave_last = r0 + 32 * wave + 31 < s.rows ? r0 + 32 * wave + 31 : s.rows - 1;
    const int wave_pos0 = s.cached + (wave_works ? (r0 + 32 * wave) / a.group : 0);
    const int wave_pos1 = s.cached + (wave_works ? wave_last / a.group : 0);
    uint4 qf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks] = make_uint4(0, 0, 0, 0);
        if (row_works)
            qf[ks] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + (int64_t)(s.start + token) * a.q_stride +
                                                      (int64_t)head * D + ks * 16 + 8 * half);
    }

    f32x16 o[D / 32], st[2];
    uint4 pf[4];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        o[db] = zero16();
    float m = -INFINITY, lsum = 0.f;
    bool seen = false;
    // What this wave moves: KEYS neighbouring keys, of V of one tile and of K of the next; this lane piece load_at of its rows,
    // from where that piece of the row is.  With WIDE, blocks of at least KEYS keys, they lie in one block: one scalar look-up,
    // uniform addresses (32768 tokens over 16384 cached 16.4 ms against 18.6 with a look-up and an address per lane).  A key that does
    // not exist is read from the cache's first rows, so that no load waits for a branch: what it gets as K comes to nothing in
    // the softmax, as V it is cleared.
    const int load_row = wave * KEYS + l / PIECES, load_at = l % PIECES;
    const SeenTiles seen_by_all(a, keys.pos0, keys.pos1, kChunkKeys), seen_by_wave(a, wave_pos0, wave_pos1, kChunkKeys);
    const int32_t *const table = reinterpret_cast<const int32_t *>(own_pointer(a.table + (int64_t)it.seq * a.max_blocks));
    const unsigned char *const k_cache = own_pointer(a.k_cache), *const v_cache = own_pointer(a.v_cache);
    const int bs_mask = (1 << a.log2_bs) - 1;
    const uint32_t lds_k_wave = lds_address(lds_k) + wave * KEYS * D * 2, lds_v_wave = lds_address(lds_v) + wave * KEYS * D * 2;
    uint32_t k_offset[LOADS], v_offset[LOADS];  // bytes behind the wave's first key's row
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = load_row + i * ROWS_PER_LOAD;
        k_offset[i] = (r - wave * KEYS) * D * 2 + ((load_at ^ Tile::k_turn(r)) << 4);
        v_offset[i] = (r - wave * KEYS) * D * 2 + ((load_at ^ Tile::v_turn(r)) << 4);
    }
    constexpr int LOOKS = WIDE ? 1 : LOADS;
    int k_row[LOOKS], v_row[LOOKS];  // WIDE: of the wave's first key, else of the lane's
#pragma unroll
    for (int i = 0; i < LOOKS; ++i)
        k_row[i] = -1;
    auto first_key = [&](int t) __attribute__((always_inline)) { return keys.tile(step_begin + t) * kChunkKeys; };
    auto look_up = [&](int j0, int (&block)[LOOKS]) __attribute__((always_inline)) {  // the blocks of a tile's keys
#pragma unroll
        for (int i = 0; i < LOOKS; ++i) {
            const int e = (j0 + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD)) >> a.log2_bs;
            const int at = (uint32_t)e < (uint32_t)a.max_blocks ? e : a.max_blocks - 1;
            block[i] = WIDE ? scalar_load(table + at) : table[at];
        }
    };
    // V of a tile, K of tile t behind it, whose first key is j0 and whose blocks have been looked up
    auto request = [&](int v_buf, int j0, const int (&block)[LOOKS], int t, int k_buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOOKS; ++i) {
            const int j = j0 + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD);
            v_row[i] = k_row[i];
            k_row[i] = j < end && (uint32_t)block[i] < (uint32_t)a.n_blocks ? ((block[i] * a.Hkv + kv_head) << a.log2_bs) + (j & bs_mask) : -1;
            // WIDE: one word for the wave's keys, else one for each; the same from all lanes of it
            lds_exist[(t & 3) * kChunkKeys + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD)] = k_row[i] >= 0;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t to_v = lds_v_wave + v_buf * Tile::kBytes + i * ROWS_PER_LOAD * D * 2, to_k = lds_k_wave + k_buf * Tile::kBytes + i * ROWS_PER_LOAD * D * 2;
            const int vr = v_row[WIDE ? 0 : i], kr = k_row[WIDE ? 0 : i];
            const unsigned char *const v = v_cache + (uint64_t)(uint32_t)(vr < 0 ? 0 : vr) * (D * 2), *const k = k_cache + (uint64_t)(uint32_t)(kr < 0 ? 0 : kr) * (D * 2);
            if (WIDE) {
                copy16_to_lds(v, v_offset[i], to_v);
                copy16_to_lds(k, k_offset[i], to_k);
            } else {
                const int own = (l / PIECES + i * ROWS_PER_LOAD) * D * 2;
                copy16_to_lds(v + v_offset[i] - own, to_v);
                copy16_to_lds(k + k_offset[i] - own, to_k);
            }
        }
    };
    auto arrive = [&](int t, int j0, int v_buf) __attribute__((always_inline)) {  // what the last request asked for, V of tile t
        memory_wait();
        const bool part_seen = !seen_by_all.all(j0);
        bool missing = WIDE && j0 + kChunkKeys > end;
#pragma unroll
        for (int i = 0; i < LOOKS; ++i)
            missing = missing || v_row[i] < 0;
        if (part_seen || __any(missing)) {
            const int l = unknown(lane_id()), load_at = l % PIECES;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = wave * KEYS + l / PIECES + i * ROWS_PER_LOAD;
                uint4 *const at = reinterpret_cast<uint4 *>(lds_v + v_buf * Tile::kBytes + r * D * 2 + load_at * 16);
                uint4 v = v_row[WIDE ? 0 : i] < 0 || j0 + r >= end ? make_uint4(0, 0, 0, 0) : *at;
                if (part_seen) {
                    bool bad = drop_not_finite<E>(v.x);
                    bad = drop_not_finite<E>(v.y) || bad;
                    bad = drop_not_finite<E>(v.z) || bad;
                    bad = drop_not_finite<E>(v.w) || bad;
                    const uint64_t of_row = __ballot(bad) >> (l / PIECES * PIECES) & ((1ull << (PIECES - 1) << 1) - 1);
                    lds_bad[(t & 3) * kChunkKeys + r] = of_row != 0;
                }
                *at = v;
            }
        }
    };
    // The operands' reads run kAhead products ahead of their use, through both products of a phase.  With the buffers known at
    // compile time their addresses differ by constants: 4 for V (2 with 64 values per head) and 8 (4) for K.
    constexpr int PV = 4 * (D / 32), QK = 2 * (D / 16), kAhead = D == 64 ? 3 : 6;
    int v_base[D / 32], k_base[D / 16];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        v_base[db] = kChunkBuffers * Tile::kBytes + Tile::v_at(4 * half + l % 16 / 4, db * 4 + 2 * (l / 16 % 2) + l % 4 / 2) + 8 * (l % 2);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        k_base[ks] = Tile::k_at(l % 32, 2 * ks + half);
    auto values = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            const unsigned char *const p = lds_raw + v_base[i % (D / 32)] + buf * Tile::kBytes + i / (D / 32) * 16 * D * 2;
            o[i % (D / 32)] = E::mfma32(lds_frag_tr(p, p + 8 * D * 2), pf[i / (D / 32)], o[i % (D / 32)]);
        }
    };
    auto scores = [&](int buf) __attribute__((always_inline)) {
        st[0] = st[1] = zero16();
#pragma unroll
        for (int i = 0; i < QK; ++i) {
            const uint4 k = *reinterpret_cast<const uint4 *>(lds_raw + k_base[i % (D / 16)] + buf * Tile::kBytes + i / (D / 16) * 32 * D * 2);
            st[i / (D / 16)] = E::mfma32(k, qf[i % (D / 16)], st[i / (D / 16)]);
        }
    };
    auto products = [&](int v_buf, int k_buf) __attribute__((always_inline)) {
        constexpr int kDsRead = 0x100, kMfma = 0x8;
        values(v_buf);
        scores(k_buf);
        __builtin_amdgcn_sched_group_barrier(kDsRead, 2 * kAhead, 0);
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
            if (i + kAhead < PV)
                __builtin_amdgcn_sched_group_barrier(kDsRead, 2, 0);
            else
                __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < QK; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
            if (i + kAhead < QK)
                __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
    };
    auto not_finite_values = [&](int t, int j0) __attribute__((always_inline)) {
        if (seen_by_all.all(j0))
            return;
        const int l = unknown(lane_id()), half = l / 32;
        const uint64_t bad = __ballot(lds_bad[(t & 3) * kChunkKeys + l] != 0);
        for (uint64_t left = bad; left != 0; left &= left - 1) {
            // V of this key has infinities or NaN, which are zeros in LDS: they go to the rows that see the key
            const int key = __builtin_ctzll(left), word = 8 * (key / 32) + 2 * (key % 32 / 8) + key % 4 / 2, from = key % 8 / 4;
            uint32_t two = 0;
#pragma unroll
            for (int w = 0; w < 16; ++w) {
                const uint4 f = pf[w / 4];
                two = w == word ? (w % 4 == 0 ? f.x : w % 4 == 1 ? f.y : w % 4 == 2 ? f.z : f.w) : two;
            }
            const float p = read_from(key % 2 ? E::hi(two) : E::lo(two), l % 32 + 32 * from);
            const int j = j0 + key, e = j >> a.log2_bs, cr = cache_row(a, j < end && e < a.max_blocks ? table[e] : -1, kv_head, j);
            const uint32_t sees_it = row_works && cr >= 0 && sees(a, pos, j) ? ~0u : 0u;
            const uint16_t *v_of = reinterpret_cast<const uint16_t *>(v_cache) + (int64_t)(cr < 0 ? 0 : cr) * D;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
                    unpack4<E>(*reinterpret_cast<const uint2 *>(v_of + db * 32 + 8 * q + 4 * half), v);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[db][4 * q + e] += not_finite_part(p, v[e], sees_it);
                }
        }
    };
    auto softmax = [&](int t, int j0) __attribute__((always_inline)) {
        const uint64_t exist = __ballot(lds_exist[(t & 3) * kChunkKeys + (WIDE ? l & -KEYS : l)] != 0);
        if (!seen_by_wave.all(j0) || exist != ~0ull) {
            const uint64_t keys_seen = seen_keys(a, unknown(pos), j0, exist);
            seen = seen || keys_seen != 0;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const uint32_t mine = (uint32_t)(keys_seen >> (32 * kb)) >> (4 * half);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    st[kb][r] = seen_score(st[kb][r], mine, 8 * (r / 4) + r % 4);
            }
        } else {
            seen = true;
        }
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                top = fmaxf(top, st[kb][r]);
        if (__any(top > m + a.outgrown)) {
            const float both = fmaxf(top, read_from(top, l ^ 32)), next = fmaxf(m, both);
            const float down = next == m ? 1.f : exp2_fast((m - next) * a.scale_log2);
            m = next;
            lsum *= down;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[db][r] *= down;
        }
        const float mc = subtrahend<E>(m, a.scale_log2);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            float p[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = exp2_fast(__builtin_fmaf(st[kb][r], a.scale_log2, -mc));
                lsum += p[r];
            }
            pf[2 * kb] = make_uint4(E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7]));
            pf[2 * kb + 1] = make_uint4(E::pack(p[8], p[9]), E::pack(p[10], p[11]), E::pack(p[12], p[13]), E::pack(p[14], p[15]));
        }
    };

    // first keys of tiles t to t + 3
    int j0 = first_key(0), j1 = first_key(1), j2 = first_key(2), j3 = first_key(3);
    int block[LOOKS], block0[LOOKS], block1[LOOKS];
    look_up(j0, block0);
    look_up(j1, block1);
    look_up(j2, block);
    request(kChunkBuffers - 1, j0, block0, 0, 0);
    request(0, j1, block1, 1, 1);
    arrive(0, j0, 0);
    lds_barrier();
    if (late)
        lds_barrier();
    if (wave_works)
        scores(0);
    auto tile = [&](int t, int buf) __attribute__((always_inline)) {  // softmax of tile t, products behind it; false behind the last tile
        const int next = (buf + 1) % kChunkBuffers, after = (buf + 2) % kChunkBuffers;
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        if (t + 1 < n)
            request(next, j2, block, t + 2, after);
        look_up(j3, block);
        if (wave_works)
            softmax(t, j0);
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        if (t + 1 >= n)
            return false;
        if (wave_works) {
            products(buf, next);
            not_finite_values(t, j0);
        }
        arrive(t + 1, j1, next);
        j0 = j1, j1 = j2, j2 = j3, j3 = first_key(t + 4);
        return true;
    };
    if (n > 0) {
        for (int t = 0; tile(t, 0) && tile(t + 1, 1) && tile(t + 2, 2); t += kChunkBuffers) {
        }
        if (wave_works) {
            values((n - 1) % kChunkBuffers);
            not_finite_values(n - 1, j0);
        }
    }
    memory_wait();
    if (!late)
        lds_barrier();
    lds_barrier();  // the last tile has been read: LDS takes the results
    if (!wave_works)
        return;
    lsum += read_from(lsum, l ^ 32);
    const int seen_there = read_from((int)seen, l ^ 32);
    const float w = row_weight(lsum, seen || seen_there != 0);
    const bool split = it.n_splits > 1;
    const int part = split ? part_of(a, it, kv_head, it.split) : 0;
    if (split && part >= a.most_parts)
        return;
    const int64_t part_row = (int64_t)part * a.rows_cap + 32 * wave;
    if (row_works && half == 0) {
        if (split)
            *reinterpret_cast<float2 *>(a.part + (int64_t)a.most_parts * a.rows_cap * D + (part_row + l % 32) * 2) = make_float2(m, w);
        else if (a.lse)
            a.lse[(int64_t)(s.start + token) * a.Hq + head] = row_lse<E>(m, w, a.scale_log2);
    }
    // A lane holds values of one row all over the head: through LDS, half of the head at a time, to rows that leave in whole lines.
    constexpr int COLS = D / 2, STRIDE = COLS + 4, LANES = COLS / 4, ROWS_AT_ONCE = 64 / LANES;
    static_assert((size_t)NW * 32 * STRIDE * sizeof(float) <= 2 * kChunkBuffers * (size_t)Tile::kBytes, "fits");
    const float scale = split ? 1.f : w == 0.f ? 0.f : w < 0.f ? NAN : 1.f / w;
    float *const mine = reinterpret_cast<float *>(lds_raw) + wave * 32 * STRIDE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        lds_wait();
#pragma unroll
        for (int db = 0; db < D / 64; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &x = o[h * (D / 64) + db];
                *reinterpret_cast<f32x4 *>(mine + l % 32 * STRIDE + db * 32 + 8 * q + 4 * half) =
                    f32x4{x[4 * q] * scale, x[4 * q + 1] * scale, x[4 * q + 2] * scale, x[4 * q + 3] * scale};
            }
        lds_wait();
#pragma unroll
        for (int i = 0; i < 32 / ROWS_AT_ONCE; ++i) {
            const int r = i * ROWS_AT_ONCE + l / LANES, d = h * COLS + l % LANES * 4;
            const f32x4 x = *reinterpret_cast<const f32x4 *>(mine + r * STRIDE + l % LANES * 4);
            const int to_token = read_from(token, r), to_head = read_from(head, r);
            if (r0 + 32 * wave + r >= s.rows)
                continue;
            if (split)
                *reinterpret_cast<f32x4 *>(a.part + (part_row + r) * D + d) = x;
            else
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + (int64_t)(s.start + to_token) * a.out_stride + (int64_t)to_head * D + d) =
                    make_uint2(E::pack(x[0], x[1]), E::pack(x[2], x[3]));
        }
    }
}

// ================================================================ few rows
// For the rows of single tokens, 16 RB of them at a time: each of the four waves takes every fourth tile of 32 keys, K from
// memory right into the operand's registers, V through LDS of its own for the transposing reads; no barriers until the waves'
// results are joined.  What bounds it is reading the cache, once: a wave's next tile is requested before the present one is used
// (64 requests over 512 to 8192 keys, 8 key heads of 128, bf16: 129 us, 5.4 TB/s; 256 with a window of 1024: 147 us, 5.2 TB/s; a
// large copy reaches 5.4, a sweep in place 6.0).  A single request over 4012 keys is latency: a call of 14 us, 8 to 10 of them
// this kernel and 5 the join.
constexpr int kFewKeys = 32;
constexpr int kFewWaves = 4;

template <int D> struct FewTile {
    static constexpr int kPieces = D / 8;
    static constexpr int kBytes = kFewKeys * D * 2;
    // V is read 16 rows at two neighbouring pieces
    static __device__ __forceinline__ int v_at(int r, int c) { return r * D * 2 + ((c ^ (D == 128 ? (r & 7) << 1 : ((r >> 1) & 3) << 1)) << 4); }
};

template <typename E, int D, int RB, bool WIDE> __global__ __launch_bounds__(64 * kFewWaves, RB * D > 128 ? 1 : 2) void attn_few_kernel(AttendArgs a)
{
    typedef FewTile<D> Tile;
    constexpr int ROWS = 16 * RB, PIECES = Tile::kPieces;
    constexpr int KS = D / 32;                         // products of a block of scores
    constexpr int V_LOADS = kFewKeys * PIECES / 64;    // pieces of V per lane
    constexpr int V_ROWS = 64 / PIECES;                // rows per such load
    extern __shared__ __align__(16) unsigned char lds_raw[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = lane_id(), quarter = l / 16;
    unsigned char *const vt = lds_raw + wave * Tile::kBytes;

    const int kv_head = blockIdx.x % a.Hkv;
    Item it;
    if (!find_item<ROWS, kFewKeys>(a, blockIdx.x / a.Hkv, false, &it))
        return;
    const Seq s = load_seq(a, it.seq);
    const int r0 = it.tile * ROWS;
    const KeyRange keys = key_range<kFewKeys>(a, s, r0, ROWS);
    const int step_begin = (int)((int64_t)keys.n * it.split / it.n_splits), step_end = (int)((int64_t)keys.n * (it.split + 1) / it.n_splits);
    const int end = keys.end;

    int pos[RB], token[RB], head[RB];
    bool row_works[RB];
    uint4 qf[RB][KS];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = r0 + 16 * rb + l % 16;
        row_works[rb] = row < s.rows;
        token[rb] = row_works[rb] ? row / a.group : 0;
        head[rb] = kv_head * a.group + (row_works[rb] ? row - token[rb] * a.group : 0);
        pos[rb] = s.cached + token[rb];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[rb][ks] = make_uint4(0, 0, 0, 0);
            if (row_works[rb])
                qf[rb][ks] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + (int64_t)(s.start + token[rb]) * a.q_stride +
                                                              (int64_t)head[rb] * D + ks * 32 + 8 * quarter);
        }
    }
    f32x4 o[RB][D / 16];
    float m[RB], lsum[RB];
    bool seen[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = -INFINITY, lsum[rb] = 0.f, seen[rb] = false;
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
            o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // With WIDE, blocks of at least 16 keys, a tile's keys lie in two blocks: scalar look-ups, and every load is a uniform address
    // and an offset that does not change (32 requests of 8 tokens, 32 rows of heads: 114 us, with a look-up per lane 126).  A key
    // that does not exist is read from the cache's first rows: as K it comes to nothing in the softmax, as V it is cleared.
    const int32_t *const table = a.table + (int64_t)it.seq * a.max_blocks;
    const int bs_mask = (1 << a.log2_bs) - 1;
    const uint32_t k_offset = l % 16 * D * 2 + 16 * quarter, v_offset = l * 16;
    constexpr int V_HALF = V_LOADS / 2;  // loads of 16 rows of V
    uint4 kreg[2][KS], vreg[V_LOADS];
    int block[2] = {-1, -1};    // of the tile behind the next: WIDE of its halves, else [0] of key l % 32
    uint32_t exist_next = 0;
    int row_of_key = -1;
    auto look_up = [&](int step) __attribute__((always_inline)) {
        const int j0 = keys.tile(step) * kFewKeys;
        if (WIDE) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = (j0 + 16 * h) >> a.log2_bs;
                block[h] = scalar_load(table + ((uint32_t)e < (uint32_t)a.max_blocks ? e : a.max_blocks - 1));
            }
        } else {
            const int e = (j0 + l % 32) >> a.log2_bs;
            block[0] = table[(uint32_t)e < (uint32_t)a.max_blocks ? e : a.max_blocks - 1];
        }
    };
    auto request = [&](int step) __attribute__((always_inline)) {
        const int j0 = keys.tile(step) * kFewKeys;
        if (WIDE) {
            exist_next = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = j0 + 16 * h;
                const bool there = j < end && (uint32_t)block[h] < (uint32_t)a.n_blocks;
                const uint32_t row = there ? (uint32_t)(((block[h] * a.Hkv + kv_head) << a.log2_bs) + (j & bs_mask)) : 0u;
                exist_next |= there ? 0xffffu << (16 * h) : 0u;
                const unsigned char *const k = static_cast<const unsigned char *>(a.k_cache) + (uint64_t)row * (D * 2);
                const unsigned char *const v = static_cast<const unsigned char *>(a.v_cache) + (uint64_t)row * (D * 2);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    kreg[h][ks] = *reinterpret_cast<const uint4 *>(k + k_offset + ks * 64);
#pragma unroll
                for (int i = 0; i < V_HALF; ++i)
                    vreg[h * V_HALF + i] = *reinterpret_cast<const uint4 *>(v + v_offset + i * 1024);
            }
            return;
        }
        const int j = j0 + l % 32;
        row_of_key = j < end && (uint32_t)block[0] < (uint32_t)a.n_blocks ? ((block[0] * a.Hkv + kv_head) << a.log2_bs) + (j & bs_mask) : -1;
        exist_next = (uint32_t)__ballot(row_of_key >= 0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const int r = read_from(row_of_key, 16 * kb + l % 16);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                kreg[kb][ks] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.k_cache) + (int64_t)(r < 0 ? 0 : r) * D + ks * 32 + 8 * quarter);
        }
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i) {
            const int r = read_from(row_of_key, i * V_ROWS + l / PIECES);
            vreg[i] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.v_cache) + (int64_t)(r < 0 ? 0 : r) * D + l % PIECES * 8);
        }
    };
    if (step_begin + wave < step_end) {
        look_up(step_begin + wave);
        request(step_begin + wave);
        look_up(step_begin + wave + kFewWaves);
    }
    const SeenTiles seen_tiles(a, keys.pos0, keys.pos1, kFewKeys);
    for (int step = step_begin + wave; step < step_end; step += kFewWaves) {
        const int j0 = keys.tile(step) * kFewKeys;
        const bool part_seen = !seen_tiles.all(j0);
        const uint32_t exist = exist_next;
        f32x4 st[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                st[rb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    st[rb][kb] = E::mfma16(kreg[kb][ks], qf[rb][ks], st[rb][kb]);
            }
        uint32_t bad = 0;  // keys whose V is not finite
        if (exist != 0xffffffffu || j0 + kFewKeys > end) {
            const int l2 = unknown(l);
#pragma unroll
            for (int i = 0; i < V_LOADS; ++i) {
                const int r = i * V_ROWS + l2 / PIECES;
                const bool there = (exist >> r & 1) != 0 && j0 + r < end;
                vreg[i] = make_uint4(there ? vreg[i].x : 0u, there ? vreg[i].y : 0u, there ? vreg[i].z : 0u, there ? vreg[i].w : 0u);
            }
        }
        if (part_seen) {
#pragma unroll
            for (int i = 0; i < V_LOADS; ++i) {
                bool b = drop_not_finite<E>(vreg[i].x);
                b = drop_not_finite<E>(vreg[i].y) || b;
                b = drop_not_finite<E>(vreg[i].z) || b;
                b = drop_not_finite<E>(vreg[i].w) || b;
                const uint64_t any = __ballot(b);
#pragma unroll
                for (int r = 0; r < V_ROWS; ++r)
                    bad |= (any >> (r * PIECES) & ((1ull << PIECES) - 1)) != 0 ? 1u << (i * V_ROWS + r) : 0u;
            }
        }
        lds_wait();  // the reads of the tile in front are done
#pragma unroll
        for (int i = 0; i < V_LOADS; ++i)
            *reinterpret_cast<uint4 *>(vt + Tile::v_at(i * V_ROWS + l / PIECES, l % PIECES)) = vreg[i];
        if (step + kFewWaves < step_end) {
            request(step + kFewWaves);
            look_up(step + 2 * kFewWaves);
        }
        const bool partly = part_seen || exist != 0xffffffffu;
        uint4 pf[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (partly) {
                const uint32_t keys_seen = (uint32_t)seen_keys(a, pos[rb], j0, exist), mine = keys_seen >> (4 * quarter);
                seen[rb] = seen[rb] || keys_seen != 0;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        st[rb][kb][r] = seen_score(st[rb][kb][r], mine, 16 * kb + r);
            } else {
                seen[rb] = true;
            }
            float top = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    top = fmaxf(top, st[rb][kb][r]);
            if (__any(top > m[rb] + a.outgrown)) {
                top = fmaxf(top, read_from(top, l ^ 16));
                top = fmaxf(top, read_from(top, l ^ 32));
                const float next = fmaxf(m[rb], top), down = next == m[rb] ? 1.f : exp2_fast((m[rb] - next) * a.scale_log2);
                m[rb] = next;
                lsum[rb] *= down;
#pragma unroll
                for (int db = 0; db < D / 16; ++db)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        o[rb][db][r] *= down;
            }
            const float mc = subtrahend<E>(m[rb], a.scale_log2);
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = exp2_fast(__builtin_fmaf(st[rb][e / 4][e % 4], a.scale_log2, -mc));
                lsum[rb] += p[e];
                st[rb][e / 4][e % 4] = p[e];
            }
            pf[rb] = make_uint4(E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7]));
        }
        lds_wait();  // V is there
        const int r_lo = 4 * quarter + (l % 16) / 4;
#pragma unroll
        for (int db = 0; db < D / 16; ++db) {
            const int c = db * 2 + (l % 4) / 2;
            const uint4 vf = lds_frag_tr(vt + Tile::v_at(r_lo, c) + 8 * (l % 2), vt + Tile::v_at(r_lo + 16, c) + 8 * (l % 2));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                o[rb][db] = E::mfma16(vf, pf[rb], o[rb][db]);
        }
        for (uint32_t left = bad; left != 0; left &= left - 1) {
            const int key = __builtin_ctz(left), e_of = 4 * (key / 16) + key % 4, from = key % 16 / 4;
            const int e = (j0 + key) >> a.log2_bs, cr = cache_row(a, j0 + key < end && e < a.max_blocks ? table[e] : -1, kv_head, j0 + key);
            const uint16_t *v_row = static_cast<const uint16_t *>(a.v_cache) + (int64_t)(cr < 0 ? 0 : cr) * D;
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                float p = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    p = e == e_of ? st[rb][e / 4][e % 4] : p;
                p = read_from(p, l % 16 + 16 * from);
                const uint32_t sees_it = row_works[rb] && cr >= 0 && sees(a, pos[rb], j0 + key) ? ~0u : 0u;
#pragma unroll
                for (int db = 0; db < D / 16; ++db) {
                    float v[4];
                    unpack4<E>(*reinterpret_cast<const uint2 *>(v_row + db * 16 + 4 * quarter), v);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[rb][db][e] += not_finite_part(p, v[e], sees_it);
                }
            }
        }
    }

    // the four waves' results, 16 rows at a time
    lds_barrier();
    float *const lds_o = reinterpret_cast<float *>(lds_raw);            // [wave][16][D + 4]
    float *const lds_ml = lds_o + kFewWaves * 16 * (D + 4);             // [wave][16][2]
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float w = lsum[rb];
        w += read_from(w, l ^ 16);
        w += read_from(w, l ^ 32);
        int any = (int)seen[rb];
        any |= read_from(any, l ^ 16);
        any |= read_from(any, l ^ 32);
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
            *reinterpret_cast<float4 *>(lds_o + (wave * 16 + l % 16) * (D + 4) + db * 16 + 4 * quarter) =
                make_float4(o[rb][db][0], o[rb][db][1], o[rb][db][2], o[rb][db][3]);
        if (quarter == 0)
            *reinterpret_cast<float2 *>(lds_ml + (wave * 16 + l) * 2) = make_float2(m[rb], row_weight(w, any != 0));
        lds_barrier();
        // thread: row tid / 16, values 4 (tid % 16) and every 64 behind them
        const int row = tid / 16, full_row = r0 + 16 * rb + row;
        if (full_row < s.rows) {
            JoinedRow j;
#pragma unroll
            for (int w2 = 0; w2 < kFewWaves; ++w2)
                j.add_max(lds_ml[(w2 * 16 + row) * 2]);
            float part_w[kFewWaves];
#pragma unroll
            for (int w2 = 0; w2 < kFewWaves; ++w2)
                part_w[w2] = j.add_weight(lds_ml[(w2 * 16 + row) * 2], lds_ml[(w2 * 16 + row) * 2 + 1], a.scale_log2);
            const int tok = full_row / a.group, hd = kv_head * a.group + full_row - tok * a.group;
            const int part = it.n_splits > 1 ? part_of(a, it, kv_head, it.split) : 0;
            if (part < a.most_parts || it.n_splits == 1) {
                const int64_t at = (int64_t)part * a.rows_cap + 16 * rb + row;
                const float scale = it.n_splits > 1 ? 1.f : j.scale();
#pragma unroll
                for (int d = 4 * (tid % 16); d < D; d += 64) {
                    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w2 = 0; w2 < kFewWaves; ++w2) {
                        const float4 x = *reinterpret_cast<const float4 *>(lds_o + (w2 * 16 + row) * (D + 4) + d);
                        if (part_w[w2] != 0.f) {
                            v[0] += part_w[w2] * x.x, v[1] += part_w[w2] * x.y, v[2] += part_w[w2] * x.z, v[3] += part_w[w2] * x.w;
                        }
                    }
                    if (it.n_splits > 1)
                        *reinterpret_cast<float4 *>(a.part + at * D + d) = make_float4(v[0], v[1], v[2], v[3]);
                    else
                        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + (int64_t)(s.start + tok) * a.out_stride + (int64_t)hd * D + d) =
                            make_uint2(E::pack(v[0] * scale, v[1] * scale), E::pack(v[2] * scale, v[3] * scale));
                }
                if (tid % 16 == 0) {
                    if (it.n_splits > 1)
                        *reinterpret_cast<float2 *>(a.part + (int64_t)a.most_parts * a.rows_cap * D + at * 2) = make_float2(j.m, j.weight());
                    else if (a.lse)
                        a.lse[(int64_t)(s.start + tok) * a.Hq + hd] = row_lse<E>(j.m, j.weight(), a.scale_log2);
                }
            }
        }
        lds_barrier();
    }
}

// ================================================================ fp32
// 16 rows per wave, 64 per workgroup, keys in tiles of 32 through LDS in two buffers; products on the fp32 matrix instructions,
// which take 2048 cycles of a wave's 4000 to 5100 per tile with heads of 64 (a sixteenth of the 16-bit rate): 3 packed prompts of
// 1537 tokens with a window of 300, 16 heads of 64, 38 us, 47 TFLOP/s; a prompt of 2000 tokens 127 us, 65 TFLOP/s.  The former is
// 392 workgroups on 256 compute units: half of them have two, and end last.  Keys from two tiles ahead, in registers, and
// addresses from scalar look-ups changed nothing.  For single tokens one of the four waves has rows.
constexpr int kF32Keys = 32;
constexpr int kF32Waves = 4;

template <int D> __global__ __launch_bounds__(64 * kF32Waves, 2) void attn_f32_kernel(AttendArgs a)
{
    constexpr int NT = 64 * kF32Waves, ROWS = 16 * kF32Waves;
    constexpr int PIECES = D / 4, LOADS = kF32Keys * PIECES / NT, ROWS_PER_LOAD = NT / PIECES;
    constexpr int STRIDE = D + 4;  // floats; rows four apart start 16 banks apart
    extern __shared__ __align__(16) unsigned char lds_raw[];
    constexpr int TILE = kF32Keys * STRIDE;
    constexpr int kAhead = 6;      // reads of V
    float *const lds_k = reinterpret_cast<float *>(lds_raw), *const lds_v = lds_k + 2 * TILE;
    int *const lds_flag = reinterpret_cast<int *>(lds_v + 2 * TILE);  // [2][32]: bit 0 the key exists, bit 1 its V is not finite

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = lane_id(), quarter = l / 16;
    const int kv_head = blockIdx.x % a.Hkv;
    Item it;
    if (!find_item<ROWS, kF32Keys>(a, blockIdx.x / a.Hkv, false, &it))
        return;
    const Seq s = load_seq(a, it.seq);
    const int r0 = it.tile * ROWS;
    const KeyRange keys = key_range<kF32Keys>(a, s, r0, ROWS);
    const int step_begin = (int)((int64_t)keys.n * it.split / it.n_splits), step_end = (int)((int64_t)keys.n * (it.split + 1) / it.n_splits);
    const int end = keys.end;

    const int row = r0 + 16 * wave + l % 16;
    const bool wave_works = r0 + 16 * wave < s.rows, row_works = row < s.rows;
    const int token = row_works ? row / a.group : 0, head = kv_head * a.group + (row_works ? row - token * a.group : 0);
    const int pos = s.cached + token;
    f32x4 qf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (row_works)
            qf[ks] = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.q) + (int64_t)(s.start + token) * a.q_stride +
                                                       (int64_t)head * D + ks * 16 + 4 * quarter);
    }
    f32x4 o[D / 16];
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
        o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, lsum = 0.f;
    bool seen = false;

    // as in the kernel for chunks: a key that does not exist is read from the cache's first row, as V it is cleared
    const int load_row = tid / PIECES, load_piece = tid % PIECES, bs_mask = (1 << a.log2_bs) - 1;
    const int32_t *const table = a.table + (int64_t)it.seq * a.max_blocks;
    f32x4 kreg[LOADS], vreg[LOADS];  // (of float4 one would be kept in memory)
    int block[LOADS], k_row[LOADS];
    auto look_up = [&](int step) __attribute__((always_inline)) {
        const int j0 = keys.tile(step) * kF32Keys + load_row;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int e = (j0 + i * ROWS_PER_LOAD) >> a.log2_bs;
            block[i] = table[(uint32_t)e < (uint32_t)a.max_blocks ? e : a.max_blocks - 1];
        }
    };
    auto request = [&](int step) __attribute__((always_inline)) {
        const int j0 = keys.tile(step) * kF32Keys + load_row;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int j = j0 + i * ROWS_PER_LOAD;
            k_row[i] = j < end && (uint32_t)block[i] < (uint32_t)a.n_blocks ? ((block[i] * a.Hkv + kv_head) << a.log2_bs) + (j & bs_mask) : -1;
            const int64_t at = (int64_t)(k_row[i] < 0 ? 0 : k_row[i]) * D + load_piece * 4;
            kreg[i] = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.k_cache) + at);
            vreg[i] = *reinterpret_cast<const f32x4 *>(static_cast<const float *>(a.v_cache) + at);
        }
    };
    if (step_begin < step_end) {
        look_up(step_begin);
        request(step_begin);
        look_up(step_begin + 1);
    }
    // q is waited for here: a wait for it in the loop would be one for the next tile's loads as well
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        qf[ks] = unknown(qf[ks]);
    const SeenTiles seen_tiles(a, keys.pos0, keys.pos1, kF32Keys);
    for (int step = step_begin; step < step_end; ++step) {
        const int j0 = keys.tile(step) * kF32Keys;
        const bool part_seen = !seen_tiles.all(j0);
        float *const kt = lds_k + (step & 1) * TILE, *const vt = lds_v + (step & 1) * TILE;
        int *const flag = lds_flag + (step & 1) * kF32Keys;
        bool missing = false;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            missing = missing || k_row[i] < 0;
        const bool clear = part_seen || __any(missing);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = load_row + i * ROWS_PER_LOAD;
            int bad = 0;
            if (clear) {
                const bool there = k_row[i] >= 0;
                uint4 v = __builtin_bit_cast(uint4, vreg[i]);
                const uint32_t all = part_seen ? 0x7f800000u : 0xffffffffu;  // what no value's exponent equals where nothing is dropped
                const bool dx = (v.x & 0x7f800000u) == all, dy = (v.y & 0x7f800000u) == all, dz = (v.z & 0x7f800000u) == all, dw = (v.w & 0x7f800000u) == all;
                const bool mine = there && (dx || dy || dz || dw);
                v = make_uint4(there && !dx ? v.x : 0u, there && !dy ? v.y : 0u, there && !dz ? v.z : 0u, there && !dw ? v.w : 0u);
                vreg[i] = __builtin_bit_cast(f32x4, v);
                bad = (__ballot(mine) >> (l / PIECES * PIECES) & ((1ull << PIECES) - 1)) != 0 ? 2 : 0;
            }
            *reinterpret_cast<f32x4 *>(kt + r * STRIDE + load_piece * 4) = kreg[i];
            *reinterpret_cast<f32x4 *>(vt + r * STRIDE + load_piece * 4) = vreg[i];
            flag[r] = (k_row[i] >= 0 ? 1 : 0) | bad;  // the same from all lanes of the row
        }
        if (step + 1 < step_end) {
            request(step + 1);
            look_up(step + 2);
        }
        lds_barrier();  // also behind the reads of the buffer that the next tile goes to
        if (!wave_works)
            continue;
        f32x4 st[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            f32x4 kf[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
                kf[kb] = *reinterpret_cast<const f32x4 *>(kt + (kb * 16 + l % 16) * STRIDE + ks * 16 + 4 * quarter);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)  // two sums in turn: a product waits for the one in front of it
                    st[kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][e], qf[ks][e], st[kb], 0, 0, 0);
        }
        const int f = flag[l % 32];
        const uint32_t exist = (uint32_t)__ballot((f & 1) != 0), bad = (uint32_t)__ballot((f & 2) != 0);
        const bool partly = part_seen || exist != 0xffffffffu;
        if (partly) {
            const uint32_t keys_seen = (uint32_t)seen_keys(a, pos, j0, exist), mine = keys_seen >> (4 * quarter);
            seen = seen || keys_seen != 0;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    st[kb][r] = seen_score(st[kb][r], mine, 16 * kb + r);
        } else {
            seen = true;
        }
        float top = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                top = fmaxf(top, st[kb][r]);
        if (__any(top > m + a.outgrown)) {
            top = fmaxf(top, read_from(top, l ^ 16));
            top = fmaxf(top, read_from(top, l ^ 32));
            const float next = fmaxf(m, top), down = next == m ? 1.f : exp2_fast((m - next) * a.scale_log2);
            m = next;
            lsum *= down;
#pragma unroll
            for (int db = 0; db < D / 16; ++db)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    o[db][r] *= down;
        }
        const float mc = subtrahend<float>(m, a.scale_log2);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = exp2_fast(__builtin_fmaf(st[e / 4][e % 4], a.scale_log2, -mc));
            lsum += p;
            st[e / 4][e % 4] = p;
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int db = 0; db < D / 16; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vt[(kb * 16 + 4 * quarter + r) * STRIDE + db * 16 + l % 16], st[kb][r], o[db], 0, 0, 0);
        // the reads of V (two of them in an instruction) run ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
            if (i + kAhead < D / 4)
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        for (uint32_t left = bad; left != 0; left &= left - 1) {
            const int key = __builtin_ctz(left), e_of = 4 * (key / 16) + key % 4, from = key % 16 / 4;
            const int e = (j0 + key) >> a.log2_bs, cr = cache_row(a, j0 + key < end && e < a.max_blocks ? table[e] : -1, kv_head, j0 + key);
            const float *v_row = static_cast<const float *>(a.v_cache) + (int64_t)(cr < 0 ? 0 : cr) * D;
            float p = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                p = e == e_of ? st[e / 4][e % 4] : p;
            p = read_from(p, l % 16 + 16 * from);
            const uint32_t sees_it = row_works && cr >= 0 && sees(a, pos, j0 + key) ? ~0u : 0u;
#pragma unroll
            for (int db = 0; db < D / 16; ++db) {
                const float4 x = *reinterpret_cast<const float4 *>(v_row + db * 16 + 4 * quarter);
                const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    o[db][e] += not_finite_part(p, v[e], sees_it);
            }
        }
    }
    if (!wave_works)
        return;
    lsum += read_from(lsum, l ^ 16);
    lsum += read_from(lsum, l ^ 32);
    int any = (int)seen;
    any |= read_from(any, l ^ 16);
    any |= read_from(any, l ^ 32);
    const float w = row_weight(lsum, any != 0);
    if (!row_works)
        return;
    const bool split = it.n_splits > 1;
    const int part = split ? part_of(a, it, kv_head, it.split) : 0;
    if (split && part >= a.most_parts)
        return;
    const int64_t at = (int64_t)part * a.rows_cap + row - r0;
    const float scale = split ? 1.f : w == 0.f ? 0.f : w < 0.f ? NAN : 1.f / w;
    float *const dst = split ? a.part + at * D : static_cast<float *>(a.out) + (int64_t)(s.start + token) * a.out_stride + (int64_t)head * D;
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
        *reinterpret_cast<float4 *>(dst + db * 16 + 4 * quarter) =
            make_float4(o[db][0] * scale, o[db][1] * scale, o[db][2] * scale, o[db][3] * scale);
    if (quarter == 0) {
        if (split)
            *reinterpret_cast<float2 *>(a.part + (int64_t)a.most_parts * a.rows_cap * D + at * 2) = make_float2(m, w);
        else if (a.lse)
            a.lse[(int64_t)(s.start + token) * a.Hq + head] = row_lse<float>(m, w, a.scale_log2);
    }
}

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

// ---------------------------------------------------------------- choice of kernels
constexpr int kChunkWaves = 8;
constexpr int kChunkRows = 32 * kChunkWaves;
constexpr int kF32Rows = 16 * kF32Waves;
constexpr int kMostFewRows = 32;

// Rows per tile, workgroups, room for partial results.
struct Launch {
    int rows;             // per tile
    uint32_t target;
    int min_steps, half_steps;
    int64_t most_tiles;   // of all sequences, per key head
    int64_t grid, join_grid, join_units, join_rows, join_blocks, parts, rows_cap;
    size_t bytes;         // of workspace
};
struct Choice {
    Launch launch;
    bool chunk;
    int row_blocks;       // of the kernel for few rows
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

// One launch for the whole batch, by the most rows that a sequence may have: each kernel takes any.  (The kernel for chunks for
// some sequences of a batch and the one for few rows for the others, a launch and a join each, lost nearly everywhere: 5
// requests of 20 to 60 tokens 30.7 us against 25.9, 64 of 1 to 512 tokens 540 against 489, of 1 to 24 221 against 226.)  Without
// a hint a batch with no more tokens than sequences is taken for single tokens.
//
// Up to 32 rows the kernel for few rows was no slower in any batch measured, and the limit is not the crossing.  With heads of 128 (one request
// over 4000 keys / 64 over up to 4000; few rows against chunks): 32 rows 21 / 97 us against 21 / 171, 48 rows 27 / 139 against 21 /
// 173, 96 rows 30 / 190 against 22 / 179.  With heads of 64 it lies behind 96 rows: 17 / 91 us against 19 / 133.  Two blocks
// of 16 rows read the keys of 17 to 32 rows once, two tiles of 16 twice: 64 requests of 32 rows 97 us against 104, but 16 such
// requests 49 against 41, one 21 against 16.  Up to 16 rows one block is never slower (one request 13, two blocks 17).
Choice choose(const attn_shape_t &s, int batch, int64_t T, int max_new)
{
    Choice c;
    const int64_t group = s.n_q_heads / s.n_kv_heads, most = max_new > 0 ? (max_new < T ? max_new : T) : T <= batch ? 1 : T, rows = most * group;
    c.row_blocks = 1;
    c.chunk = false;
    if (s.io_dtype == ATTN_DT_F32) {
        c.launch = make_launch(s, batch, T, kF32Rows, 1024, 10, 32);  // (a prompt of 2000 tokens 127 us, shared by 512 137)
    } else if (rows <= kMostFewRows) {
        c.row_blocks = rows <= 16 ? 1 : 2;
        // Many small pieces balance long batches, but each costs the wait for its first keys and a partial result: 64 requests over 512 to
        // 8192 keys 136 us (shared by 512 workgroups 145), 32 with a single key head 32 us, 16 of up to 5 tokens 30 (always by 1024 37, 34).
        c.launch = make_launch(s, batch, T, 16 * c.row_blocks, 1024, 4, 24);
    } else {
        c.chunk = true;
        // Partial results of less than a tile's rows cost little: 32 requests of 16 tokens with 64 rows of heads 116 us, shared by 256
        // workgroups 172 (16 of 56 tokens 80, 72).  Those of whole tiles cost more than the balance gives: a prompt of 2000 tokens
        // 88 us shared by 512, 61 by 256, 4 of 500 to 1500 tokens 49, 46 (16 of 80 to 128 tokens 98 to 123, 136 to 140).
        c.launch = rows < kChunkRows ? make_launch(s, batch, T, kChunkRows, 512, 6, 16) : make_launch(s, batch, T, kChunkRows, 256, 6, 0);
    }
    return c;
}

// The most steps of KT keys that a tile of `rows` rows can have in a table of this width: fewer than one and a half times
// min_steps are never split.
template <int KT> bool may_split(const AttendArgs &a, const Launch &c)
{
    int64_t steps = ((((int64_t)a.max_blocks << a.log2_bs) + KT - 1) / KT);
    if (a.window > 0) {
        const int64_t seen = ((int64_t)a.window + c.rows / a.group + 1) / KT + 2 + ((int64_t)a.sinks + KT - 1) / KT;
        steps = seen < steps ? seen : steps;
    }
    return steps + c.min_steps / 2 >= 2 * (int64_t)c.min_steps;
}

template <typename E, int D> hipError_t join(const AttendArgs &a, const Launch &c, bool few, bool f32, hipStream_t stream)
{
    if (c.join_grid == 0 || !(f32 ? may_split<kF32Keys>(a, c) : few ? may_split<kFewKeys>(a, c) : may_split<kChunkKeys>(a, c)))
        return hipSuccess;
    const dim3 grid((unsigned)c.join_grid), block(kJoinThreads);
    if (f32)
        hipLaunchKernelGGL((attn_join_kernel<float, D, kF32Rows, kF32Keys>), grid, block, 0, stream, a, (int)c.join_rows, (int)c.join_blocks, (int)c.join_grid, (int)c.join_units);
    else if (!few)
        hipLaunchKernelGGL((attn_join_kernel<E, D, kChunkRows, kChunkKeys>), grid, block, 0, stream, a, (int)c.join_rows, (int)c.join_blocks, (int)c.join_grid, (int)c.join_units);
    else if (c.rows == 16)
        hipLaunchKernelGGL((attn_join_kernel<E, D, 16, kFewKeys>), grid, block, 0, stream, a, (int)c.join_rows, (int)c.join_blocks, (int)c.join_grid, (int)c.join_units);
    else
        hipLaunchKernelGGL((attn_join_kernel<E, D, 32, kFewKeys>), grid, block, 0, stream, a, (int)c.join_rows, (int)c.join_blocks, (int)c.join_grid, (int)c.join_units);
    return hipGetLastError();
}

template <typename K> hipError_t lds_limit(K kernel, size_t lds)
{
    return lds > 65536 ? hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)
                       : hipSuccess;
}

template <typename E, int D, int RB> hipError_t launch_few(const AttendArgs &a, const Launch &c, hipStream_t stream)
{
    constexpr size_t v = (size_t)kFewWaves * FewTile<D>::kBytes, o = (size_t)kFewWaves * 16 * (D + 4 + 2) * sizeof(float);
    constexpr size_t lds = v > o ? v : o;
    if (1 << a.log2_bs >= 16)
        hipLaunchKernelGGL((attn_few_kernel<E, D, RB, true>), dim3((unsigned)c.grid), dim3(64 * kFewWaves), lds, stream, a);
    else
        hipLaunchKernelGGL((attn_few_kernel<E, D, RB, false>), dim3((unsigned)c.grid), dim3(64 * kFewWaves), lds, stream, a);
    return hipGetLastError();
}

template <typename E, int D> hipError_t launch16(const AttendArgs &a, const Launch &c, bool chunk, hipStream_t stream)
{
    hipError_t e;
    if (chunk) {
        constexpr size_t lds = 2 * kChunkBuffers * (size_t)ChunkTile<D>::kBytes + 8 * kChunkKeys * sizeof(int);
        const bool wide = 1 << a.log2_bs >= kChunkKeys / kChunkWaves;
        e = wide ? lds_limit(attn_chunk_kernel<E, D, kChunkWaves, true>, lds) : lds_limit(attn_chunk_kernel<E, D, kChunkWaves, false>, lds);
        if (e != hipSuccess)
            return e;
        if (wide)
            hipLaunchKernelGGL((attn_chunk_kernel<E, D, kChunkWaves, true>), dim3((unsigned)c.grid), dim3(64 * kChunkWaves), lds, stream, a);
        else
            hipLaunchKernelGGL((attn_chunk_kernel<E, D, kChunkWaves, false>), dim3((unsigned)c.grid), dim3(64 * kChunkWaves), lds, stream, a);
        e = hipGetLastError();
    } else {
        e = c.rows == 16 ? launch_few<E, D, 1>(a, c, stream) : launch_few<E, D, 2>(a, c, stream);
    }
    return e != hipSuccess ? e : join<E, D>(a, c, !chunk, false, stream);
}

template <int D> hipError_t launch_f32(const AttendArgs &a, const Launch &c, hipStream_t stream)
{
    constexpr size_t lds = 4 * (size_t)kF32Keys * (D + 4) * sizeof(float) + 2 * kF32Keys * sizeof(int);
    const hipError_t limit = lds_limit(attn_f32_kernel<D>, lds);
    if (limit != hipSuccess)
        return limit;
    hipLaunchKernelGGL((attn_f32_kernel<D>), dim3((unsigned)c.grid), dim3(64 * kF32Waves), lds, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : join<float, D>(a, c, false, true, stream);
}

}  // namespace

size_t attn_attend_workspace(const attn_shape_t &s, int batch, int64_t T, int max_new)
{
    if (T == 0 || batch == 0)
        return 0;
    return choose(s, batch, T, max_new).launch.bytes;
}

hipError_t launch_attn_attend(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, const void *q,
                              int64_t q_stride, const void *k_cache, const void *v_cache, const int32_t *table,
                              const int32_t *cu, const int32_t *cached, float scale, int window, int sinks, int max_new,
                              void *out, int64_t out_stride, float *lse, void *workspace, hipStream_t stream)
{
    const Choice c = choose(s, batch, T, max_new);
    const Launch &u = c.launch;
    if (u.grid > 0x7fffffff || u.join_units > 0x7fffffff - kJoinWorkgroups)
        return hipErrorInvalidValue;
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
    if (s.io_dtype == ATTN_DT_F32)
        return s.head_dim == 64 ? launch_f32<64>(a, u, stream) : launch_f32<128>(a, u, stream);
    if (s.io_dtype == ATTN_DT_BF16)
        return s.head_dim == 64 ? launch16<Bf16, 64>(a, u, c.chunk, stream) : launch16<Bf16, 128>(a, u, c.chunk, stream);
    return s.head_dim == 64 ? launch16<F16, 64>(a, u, c.chunk, stream) : launch16<F16, 128>(a, u, c.chunk, stream);
}
