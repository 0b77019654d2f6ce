// Attention of drafted trees: more rows than single tokens have, fewer than chunks, over long caches.  Formulas, layouts of the products
// and the treatment of what is not finite are those of attn_attend.hip.
//
// Up to some 200 rows per key head reading the cache bounds (a row is 1 operation per byte and value, the machine's balance 260),
// so what counts is bytes on their way.  A workgroup of NW waves takes 32 rows per wave and walks the keys in tiles of 32, K and V
// in LDS in three buffers each of 8 KB (128 values per head): two tiles are on their way while one is worked on, and three
// workgroups, 96 KB on their way, share a compute unit; their products and softmaxes run under one another without any
// order between them.  One barrier per tile.
#include "attn_common.h"
#include "attn_join.h"

namespace {

template <typename E> __device__ __forceinline__ void unpack4(uint2 u, float *v)
{
    v[0] = E::lo(u.x), v[1] = E::hi(u.x), v[2] = E::lo(u.y), v[3] = E::hi(u.y);
}

// All of the wave's copies but the last N have arrived.
template <int N> __device__ __forceinline__ void memory_wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

constexpr int kTreeKeys = 32;
constexpr int kTreeBuffers = 3;

template <int D> struct TreeTile {
    static constexpr int kPieces = D / 8;  // 16-byte pieces of a row
    static constexpr int kBytes = kTreeKeys * D * 2;
    // as the chunks' tiles: K is read 32 rows at a piece, V 8 rows at four neighbouring pieces
    static __device__ __forceinline__ int k_turn(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_turn(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
    static __device__ __forceinline__ int k_at(int r, int c) { return r * D * 2 + ((c ^ k_turn(r)) << 4); }
    static __device__ __forceinline__ int v_at(int r, int c) { return r * D * 2 + ((c ^ v_turn(r)) << 4); }
};
template <int D, int NW> constexpr size_t tree_lds()
{
    constexpr size_t tiles = 2 * kTreeBuffers * (size_t)TreeTile<D>::kBytes, out = (size_t)NW * 32 * (D / 2 + 4) * sizeof(float);
    return (tiles > out ? tiles : out) + 8 * kTreeKeys * sizeof(int);
}

// WIDE: the keys that a wave moves lie in one block.
template <typename E, int D, int NW, bool WIDE> __global__ __launch_bounds__(64 * NW, D == 64 ? 4 : NW == 4 ? 3 : 2) void attn_tree_kernel(AttendArgs a)
{
    typedef TreeTile<D> Tile;
    constexpr int ROWS = 32 * NW, PIECES = Tile::kPieces;
    constexpr int KEYS = kTreeKeys / NW;       // of a tile, that a wave moves
    constexpr int LOADS = KEYS * PIECES / 64;  // copies of K (and of V) for them
    constexpr int ROWS_PER_LOAD = 64 / PIECES;
    static_assert(LOADS >= 1 && LOADS * ROWS_PER_LOAD == KEYS, "whole copies");
    extern __shared__ __align__(16) unsigned char lds_raw[];
    unsigned char *const lds_k = lds_raw, *const lds_v = lds_raw + kTreeBuffers * Tile::kBytes;
    // of four tiles: which keys exist, and whose V is not finite
    int *const lds_exist = reinterpret_cast<int *>(lds_raw + tree_lds<D, NW>() - 8 * kTreeKeys * sizeof(int)), *const lds_bad = lds_exist + 4 * kTreeKeys;

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), l = lane_id(), half = l / 32;
    const int kv_head = blockIdx.x % a.Hkv;
    Item it;
    if (!find_item<ROWS, kTreeKeys>(a, blockIdx.x / a.Hkv, false, &it))
        return;
    const Seq s = load_seq(a, it.seq);
    const int r0 = it.tile * ROWS;
    const KeyRange keys = key_range<kTreeKeys, true>(a, s, r0, ROWS);
    const int step_begin = (int)((int64_t)keys.n * it.split / it.n_splits);
    const int n = (int)((int64_t)keys.n * (it.split + 1) / it.n_splits) - step_begin;
    const int end = keys.end;

    // this lane's row
    const int row = r0 + 32 * wave + l % 32;
    const bool wave_works = r0 + 32 * wave < s.rows, row_works = row < s.rows;
    const int token = row_works ? row / a.group : 0, head = kv_head * a.group + (row_works ? row - token * a.group : 0);
    int pos = row_works ? tree_position(a, s, token) : s.cached;
    uint4 qf[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks] = make_uint4(0, 0, 0, 0);
        if (row_works)
            qf[ks] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + (int64_t)(s.start + token) * a.q_stride +
                                                      (int64_t)head * D + ks * 16 + 8 * half);
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        o[db] = zero16();
    float m = -INFINITY, lsum = 0.f;
    bool seen = false;
    const SeenTiles seen_by_all(a, keys.pos0 - 1, keys.pos1, kTreeKeys);

    // A key that does not exist is read from the cache's first rows: as K it comes to nothing in the softmax, as V it is cleared.
    const int load_row = wave * KEYS + l / PIECES, load_at = l % PIECES;
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
    int rows_of[kTreeBuffers][LOOKS];  // of the present tile and the next ones; WIDE: of the wave's first key, else of the lane's
    auto first_key = [&](int t) __attribute__((always_inline)) { return keys.tile(step_begin + t) * kTreeKeys; };
    auto look_up = [&](int j0, int (&block)[LOOKS]) __attribute__((always_inline)) {  // the blocks of a tile's keys
#pragma unroll
        for (int i = 0; i < LOOKS; ++i) {
            const int e = (j0 + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD)) >> a.log2_bs;
            const int at = (uint32_t)e < (uint32_t)a.max_blocks ? e : a.max_blocks - 1;
            block[i] = WIDE ? scalar_load(table + at) : table[at];
        }
    };
    // K and V of tile t, whose first key is j0 and whose blocks have been looked up
    auto request = [&](int t, int j0, const int (&block)[LOOKS], int (&rows)[LOOKS], int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LOOKS; ++i) {
            const int j = j0 + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD);
            rows[i] = j < end && (uint32_t)block[i] < (uint32_t)a.n_blocks ? ((block[i] * a.Hkv + kv_head) << a.log2_bs) + (j & bs_mask) : -1;
            // WIDE: one word for the wave's keys, else one for each; the same from all lanes of it
            lds_exist[(t & 3) * kTreeKeys + (WIDE ? wave * KEYS : load_row + i * ROWS_PER_LOAD)] = rows[i] >= 0;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t to_v = lds_v_wave + buf * Tile::kBytes + i * ROWS_PER_LOAD * D * 2, to_k = lds_k_wave + buf * Tile::kBytes + i * ROWS_PER_LOAD * D * 2;
            const int r = rows[WIDE ? 0 : i];
            const uint64_t at = (uint64_t)(uint32_t)(r < 0 ? 0 : r) * (D * 2);
            if (WIDE) {
                copy16_to_lds(k_cache + at, k_offset[i], to_k);
                copy16_to_lds(v_cache + at, v_offset[i], to_v);
            } else {
                const int own = (l / PIECES + i * ROWS_PER_LOAD) * D * 2;
                copy16_to_lds(k_cache + at + k_offset[i] - own, to_k);
                copy16_to_lds(v_cache + at + v_offset[i] - own, to_v);
            }
        }
    };
    // Tile t, whose copies have arrived: V of keys that do not exist becomes zeros; so do infinities and NaN where not every row sees
    // every key.
    auto clean = [&](int t, int j0, const int (&rows)[LOOKS], int buf) __attribute__((always_inline)) {
        const bool part_seen = !seen_by_all.all(j0);
        bool missing = WIDE && j0 + kTreeKeys > end;
#pragma unroll
        for (int i = 0; i < LOOKS; ++i)
            missing = missing || rows[i] < 0;
        if (part_seen || __any(missing)) {
            const int l = unknown(lane_id()), load_at = l % PIECES;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = wave * KEYS + l / PIECES + i * ROWS_PER_LOAD;
                uint4 *const at = reinterpret_cast<uint4 *>(lds_v + buf * Tile::kBytes + r * D * 2 + load_at * 16);
                uint4 v = rows[WIDE ? 0 : i] < 0 || j0 + r >= end ? make_uint4(0, 0, 0, 0) : *at;
                if (part_seen) {
                    bool bad = drop_not_finite<E>(v.x);
                    bad = drop_not_finite<E>(v.y) || bad;
                    bad = drop_not_finite<E>(v.z) || bad;
                    bad = drop_not_finite<E>(v.w) || bad;
                    const uint64_t of_row = __ballot(bad) >> (l / PIECES * PIECES) & ((1ull << (PIECES - 1) << 1) - 1);
                    lds_bad[(t & 3) * kTreeKeys + r] = of_row != 0;
                }
                *at = v;
            }
        }
    };
    int v_base[D / 32], k_base[D / 16];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
        v_base[db] = kTreeBuffers * Tile::kBytes + Tile::v_at(4 * half + l % 16 / 4, db * 4 + 2 * (l / 16 % 2) + l % 4 / 2) + 8 * (l % 2);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        k_base[ks] = Tile::k_at(l % 32, 2 * ks + half);
    auto work = [&](int t, int j0, int buf) __attribute__((always_inline)) {
        f32x16 st = zero16();
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
            st = E::mfma32(*reinterpret_cast<const uint4 *>(lds_raw + k_base[ks] + buf * Tile::kBytes), qf[ks], st);
        const bool part_seen = !seen_by_all.all(j0);
        const uint32_t exist = (uint32_t)__ballot(lds_exist[(t & 3) * kTreeKeys + (WIDE ? l % 32 & -KEYS : l % 32)] != 0);
        if (part_seen || exist != ~0u) {
            const uint32_t keys_seen = (uint32_t)seen_keys<true>(a, s, unknown(pos), unknown(token), j0, exist), mine = keys_seen >> (4 * half);
            seen = seen || keys_seen != 0;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                st[r] = seen_score(st[r], mine, 8 * (r / 4) + r % 4);
        } else {
            seen = true;
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            top = fmaxf(top, st[r]);
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
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = exp2_fast(__builtin_fmaf(st[r], a.scale_log2, -mc));
            lsum += p[r];
        }
        const uint4 pf[2] = {make_uint4(E::pack(p[0], p[1]), E::pack(p[2], p[3]), E::pack(p[4], p[5]), E::pack(p[6], p[7])),
                             make_uint4(E::pack(p[8], p[9]), E::pack(p[10], p[11]), E::pack(p[12], p[13]), E::pack(p[14], p[15]))};
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                const unsigned char *const v = lds_raw + v_base[db] + buf * Tile::kBytes + ks * 16 * D * 2;
                o[db] = E::mfma32(lds_frag_tr(v, v + 8 * D * 2), pf[ks], o[db]);
            }
        if (!part_seen)
            return;
        const int l = unknown(lane_id()), half = l / 32;
        const uint32_t bad = (uint32_t)__ballot(lds_bad[(t & 3) * kTreeKeys + l % 32] != 0);
        for (uint32_t left = bad; left != 0; left &= left - 1) {
            // V of this key has infinities or NaN, which are zeros in LDS: they go to the rows that see the key
            const int key = __builtin_ctz(left), word = 2 * (key / 8) + key % 4 / 2, from = key % 8 / 4;
            uint32_t two = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const uint4 f = pf[w / 4];
                two = w == word ? (w % 4 == 0 ? f.x : w % 4 == 1 ? f.y : w % 4 == 2 ? f.z : f.w) : two;
            }
            const float weight = read_from(key % 2 ? E::hi(two) : E::lo(two), l % 32 + 32 * from);
            const int j = j0 + key, e = j >> a.log2_bs, cr = cache_row(a, j < end && e < a.max_blocks ? table[e] : -1, kv_head, j);
            const uint32_t sees_it = row_works && cr >= 0 && sees<true>(a, s, pos, token, j) ? ~0u : 0u;
            const uint16_t *const v_of = reinterpret_cast<const uint16_t *>(v_cache) + (int64_t)(cr < 0 ? 0 : cr) * D;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
                    unpack4<E>(*reinterpret_cast<const uint2 *>(v_of + db * 32 + 8 * q + 4 * half), v);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[db][4 * q + e] += not_finite_part(weight, v[e], sees_it);
                }
        }
    };

    int j0 = first_key(0), j1 = first_key(1), j2 = first_key(2);
    int block[LOOKS];
    if (n > 0) {
        int block0[LOOKS], block1[LOOKS];
        look_up(j0, block0);
        look_up(j1, block1);
        look_up(j2, block);
        request(0, j0, block0, rows_of[0], 0);
        if (n > 1)
            request(1, j1, block1, rows_of[1], 1);
    }
    // q and positions are waited for here: a wait for them in the loop would be one for the copies on their way as well
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        qf[ks].x = unknown(qf[ks].x), qf[ks].y = unknown(qf[ks].y), qf[ks].z = unknown(qf[ks].z), qf[ks].w = unknown(qf[ks].w);
    pos = unknown(pos);
    auto tile = [&](int t, int buf) __attribute__((always_inline)) {  // false behind the last tile
        constexpr int OF_TILE = 2 * LOADS;
        if (t + 1 < n && WIDE)
            memory_wait_but<OF_TILE>();
        else
            memory_wait();
        clean(t, j0, rows_of[buf], buf);
        lds_barrier();  // the tile is there, and the one in front has been read by all
        const int after = (buf + 2) % kTreeBuffers;
        if (t + 2 < n)
            request(t + 2, j2, block, rows_of[after], after);
        const int j3 = first_key(t + 3);
        look_up(j3, block);
        if (wave_works)
            work(t, j0, buf);
        j0 = j1, j1 = j2, j2 = j3;
        return t + 1 < n;
    };
    if (n > 0)
        for (int t = 0; tile(t, 0) && tile(t + 1, 1) && tile(t + 2, 2); t += kTreeBuffers) {
        }
    memory_wait();
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

// ---------------------------------------------------------------- choice of kernels
struct TreeChoice {
    Launch launch;
    int waves;  // 0: a kernel of attn_attend.hip
};
// By the most rows that a sequence may have (us, times against those of the kernels of attn_attend.hip; 32 heads and 8 key heads of 128
// values in bf16, 32 trees over 114453 cached keys in all, 64 over 136644, 8 over 27462):  up to 32 the kernel for few rows is faster
// anyway;  up to 64 two waves (32 trees of 8 to 16 tokens 117, 146);  up to 128 four (64 trees of 32 tokens 171, 215; one of 17 over
// 4011 keys 20.5, 22.1);  up to 256 two tiles of four waves, whose keys come from memory once and from the L2 again, where there are
// sequences and key heads for every compute unit (32 trees of 16 to 64 tokens 162, 229; others over 86418 keys 119), else the kernel
// for chunks (8 trees of 64 tokens 66, 57; one 37, 32), as for more rows.
//
// A partial result of 64 rows costs as much memory time as 4 tiles: where sequences and key heads alone are work enough, pieces get at
// least 24 tiles (32 trees of 16 to 64 tokens 162, with 8 and shared by 768 workgroups 188), else 6.  Four waves are shared by 400
// workgroups, half of what may run at once, as their partial results are twice as large (64 trees of 32 tokens 171, by 640 186).
TreeChoice choose_tree(const attn_shape_t &s, int batch, int64_t T, int max_new)
{
    TreeChoice c;
    const int64_t group = s.n_q_heads / s.n_kv_heads, most = max_new > 0 && max_new < T ? max_new : T, rows = most * group;
    const bool many = (int64_t)(batch < T ? batch : T) * s.n_kv_heads >= 256;
    c.waves = s.io_dtype == ATTN_DT_F32 || rows <= 32 ? 0 : rows <= 64 ? 2 : rows <= 128 || (rows <= 256 && many) ? 4 : 0;
    if (c.waves) {
        const bool fine = many && (rows <= 64 || rows > 128);
        c.launch = make_launch(s, batch, T, 32 * c.waves, c.waves == 4 && rows <= 128 ? 400 : 640, fine ? 24 : 6, fine ? 0 : 24);
        // most tiles are cut here: as many workgroups for the joins as there are rows for (64 trees of 32 tokens 186, by 256 workgroups 201)
        c.launch.join_grid = c.launch.join_units < kJoinWorkgroups ? c.launch.join_units : kJoinWorkgroups;
    }
    return c;
}

template <typename E, int D, int NW> hipError_t launch_waves(const AttendArgs &a, const Launch &c, hipStream_t stream)
{
    hipError_t e = 1 << a.log2_bs >= kTreeKeys / NW ? launch_on(attn_tree_kernel<E, D, NW, true>, a, c, 64 * NW, tree_lds<D, NW>(), stream)
                                                    : launch_on(attn_tree_kernel<E, D, NW, false>, a, c, 64 * NW, tree_lds<D, NW>(), stream);
    if (e != hipSuccess || c.join_grid == 0 || !may_split<kTreeKeys>(a, c))
        return e;
    hipLaunchKernelGGL((attn_join_kernel<E, D, 32 * NW, kTreeKeys>), dim3((unsigned)c.join_grid), dim3(kJoinThreads), 0, stream, a, (int)c.join_rows, (int)c.join_blocks,
                       (int)c.join_grid, (int)c.join_units);
    return hipGetLastError();
}

template <typename E> hipError_t launch_dim(const attn_shape_t &s, const AttendArgs &a, const TreeChoice &c, hipStream_t stream)
{
    if (s.head_dim == 64)
        return c.waves == 2 ? launch_waves<E, 64, 2>(a, c.launch, stream) : launch_waves<E, 64, 4>(a, c.launch, stream);
    return c.waves == 2 ? launch_waves<E, 128, 2>(a, c.launch, stream) : launch_waves<E, 128, 4>(a, c.launch, stream);
}

}  // namespace

size_t attn_attend_tree_workspace(const attn_shape_t &s, int batch, int64_t T, int max_new)
{
    if (T == 0 || batch == 0)
        return 0;
    const TreeChoice c = choose_tree(s, batch, T, max_new);
    return c.waves ? c.launch.bytes : attn_attend_workspace(s, batch, T, max_new);
}

hipError_t launch_attn_attend_tree(const attn_shape_t &s, int batch, int64_t T, int n_blocks, int max_blocks, const void *q,
                                   int64_t q_stride, const void *k_cache, const void *v_cache, const int32_t *table,
                                   const int32_t *cu, const int32_t *cached, float scale, int window, int sinks, int max_new,
                                   void *out, int64_t out_stride, float *lse, void *workspace, hipStream_t stream, const AttnTrees &trees)
{
    const TreeChoice c = choose_tree(s, batch, T, max_new);
    if (!c.waves)
        return launch_attn_attend(s, batch, T, n_blocks, max_blocks, q, q_stride, k_cache, v_cache, table, cu, cached, scale, window, sinks, max_new, out, out_stride, lse,
                                  workspace, stream, trees);
    const Launch &u = c.launch;
    if (u.grid > 0x7fffffff || u.join_units > 0x7fffffff - kJoinWorkgroups)
        return hipErrorInvalidValue;
    AttendArgs a = attend_args(s, batch, T, n_blocks, max_blocks, q, q_stride, k_cache, v_cache, table, cu, cached, scale, window, sinks, out, out_stride, lse, workspace, u);
    a.positions = trees.positions;
    a.seen = trees.seen;
    a.words = trees.words;
    if (s.io_dtype == ATTN_DT_BF16)
        return launch_dim<Bf16>(s, a, c, stream);
    return launch_dim<F16>(s, a, c, stream);
}
