// Driver of the CPU emulation for the attention operators (test infrastructure only): reads a problem file, runs the
// CPU-compiled kernels on fibers through their launchers and writes what they wrote.  Every buffer has its exact size and
// sits flush against an inaccessible page.
//   emu_attn_main <in.bin> <out.bin> [order] [end|start]
// The problem: a magic word, the operator, 32 parameters, then the arrays in the order in which they are read here.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <vector>

#include "attn_common.h"
#include "emu_host.h"

namespace emu {
void set_order_mode(int m);
long switches();
}  // namespace emu

static bool g_end = true;
static FILE *g_in;

template <typename T> static T *array(size_t n)
{
    T *p = static_cast<T *>(guarded((n ? n : 1) * sizeof(T), g_end));
    read_vec(g_in, p, n);
    return p;
}
static unsigned char *blank(size_t bytes)
{
    unsigned char *p = static_cast<unsigned char *>(guarded(bytes ? bytes : 1, g_end));
    memset(p, 0xFF, bytes);  // NaN patterns: every output must be written
    return p;
}

int main(int argc, char **argv)
{
    if (argc < 3)
        return 2;
    emu::set_order_mode(argc > 3 ? atoi(argv[3]) : 0);
    g_end = !(argc > 4 && argv[4][0] == 's');
    g_in = fopen(argv[1], "rb");
    if (!g_in)
        return 2;
    int32_t h[34];
    read_vec(g_in, h, 34);
    if (h[0] != 0x4154544e)
        return 2;
    const int32_t *p = h + 2;
    FILE *out = fopen(argv[2], "wb");
    hipError_t e = hipSuccess;
    if (h[1] == 0) {  // assign
        const int batch = p[0], log2_bs = p[1], max_blocks = p[2], T = p[3], has_shared = p[4], capacity = p[5], in_place = p[6];
        int32_t *cu = array<int32_t>(batch + 1), *cached = array<int32_t>(batch), *shared = has_shared ? array<int32_t>(batch) : nullptr;
        int32_t *table = array<int32_t>((size_t)batch * max_blocks), *free_blocks = array<int32_t>(capacity), *n_free = array<int32_t>(1);
        int32_t *table_out = in_place ? table : reinterpret_cast<int32_t *>(blank((size_t)batch * max_blocks * 4));
        int64_t *slots = reinterpret_cast<int64_t *>(blank((size_t)T * 8));
        int32_t *positions = reinterpret_cast<int32_t *>(blank((size_t)T * 4)), *copies = reinterpret_cast<int32_t *>(blank((size_t)batch * 16));
        int32_t *counts = reinterpret_cast<int32_t *>(blank(8));
        e = launch_attn_assign(batch, log2_bs, max_blocks, T, cu, cached, shared, table, table_out, free_blocks, n_free, capacity, slots,
                               positions, copies, counts, nullptr);
        fwrite(table_out, 4, (size_t)batch * max_blocks, out);
        fwrite(slots, 8, T, out);
        fwrite(positions, 4, T, out);
        fwrite(copies, 16, batch, out);
        fwrite(counts, 4, 2, out);
    } else {
        attn_shape_t s;
        s.n_q_heads = p[0], s.n_kv_heads = p[1], s.head_dim = p[2], s.block_size = p[3], s.io_dtype = p[4];
        const size_t esz = s.io_dtype == ATTN_DT_F32 ? 4 : 2;
        const int T = p[5], batch = p[6], n_blocks = p[7];
        const size_t cache = (size_t)n_blocks * s.n_kv_heads * s.block_size * s.head_dim * esz;
        if (h[1] == 1) {  // rope
            const int max_positions = p[8], rot = p[9], interleaved = p[10], has_copies = p[11], row = p[12];  // row: elements of a token of q, k, v together
            unsigned char *qkv = array<unsigned char>((size_t)T * row * esz);
            int32_t *positions = array<int32_t>(T);
            int64_t *slots = array<int64_t>(T);
            float *rotary = array<float>((size_t)max_positions * rot);
            int32_t *copies = has_copies ? array<int32_t>((size_t)batch * 4) : nullptr;
            unsigned char *k_cache = array<unsigned char>(cache), *v_cache = array<unsigned char>(cache);
            const size_t q_bytes = (size_t)s.n_q_heads * s.head_dim * esz, k_bytes = (size_t)s.n_kv_heads * s.head_dim * esz;
            unsigned char *q_out = blank((size_t)T * q_bytes);
            e = launch_attn_rope(s, T, batch, n_blocks, qkv, row, qkv + q_bytes, row, qkv + q_bytes + k_bytes, row, positions, slots,
                                 rotary, max_positions, rot, interleaved != 0, copies, q_out, k_cache, v_cache, nullptr);
            fwrite(q_out, 1, (size_t)T * q_bytes, out);
            fwrite(k_cache, 1, cache, out);
            fwrite(v_cache, 1, cache, out);
        } else {  // attend
            const int max_blocks = p[8], window = p[9], sinks = p[10], max_new = p[11], q_row = p[13];
            float scale;
            memcpy(&scale, p + 12, 4);
            // the last token's row ends with its heads, also where rows are farther apart
            const size_t row = (size_t)s.n_q_heads * s.head_dim, q_n = T ? (size_t)(T - 1) * q_row + row : 0;
            unsigned char *q = array<unsigned char>(q_n * esz), *k = array<unsigned char>(cache), *v = array<unsigned char>(cache);
            int32_t *table = array<int32_t>((size_t)batch * max_blocks), *cu = array<int32_t>(batch + 1), *cached = array<int32_t>(batch);
            unsigned char *o = blank((size_t)T * row * esz);
            float *lse = reinterpret_cast<float *>(blank((size_t)T * s.n_q_heads * 4));
            unsigned char *ws = blank(attn_attend_workspace(s, batch, T, max_new));
            e = launch_attn_attend(s, batch, T, n_blocks, max_blocks, q, q_row, k, v, table, cu, cached, scale, window, sinks, max_new,
                                   o, row, lse, ws, nullptr);
            fwrite(o, 1, (size_t)T * row * esz, out);
            fwrite(lse, 4, (size_t)T * s.n_q_heads, out);
        }
    }
    fclose(out);
    if (e != hipSuccess) {
        fprintf(stderr, "launch failed: %d\n", e);
        return 4;
    }
    printf("emu ok: %ld fiber switches\n", emu::switches());
    return 0;
}
