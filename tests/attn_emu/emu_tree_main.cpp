// Driver of the CPU emulation for the operators of steps with trees (test infrastructure only); the manner is emu_attn_main.cpp's.
//   emu_tree_main <in.bin> <out.bin> [order] [end|start]
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <vector>

#include "attn_common.h"
#include "emu_host.h"

namespace emu {
void set_order_mode(int m);
}  // namespace emu

static bool g_end = true;
static FILE *g_in;

template <typename T> static T *array(size_t n)
{
    T *p = static_cast<T *>(guarded((n ? n : 1) * sizeof(T), g_end));
    read_vec(g_in, p, n);
    return p;
}
template <typename T> static T *blank(size_t n)
{
    T *p = static_cast<T *>(guarded((n ? n : 1) * sizeof(T), g_end));
    memset(p, 0xA5, n * sizeof(T));  // every output must be written
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
    const int batch = p[0], T = p[1];
    int32_t *cu = array<int32_t>(batch + 1), *cached = array<int32_t>(batch);
    if (h[1] == 0) {  // draft_tree
        const int words = p[2];
        int32_t *parents = array<int32_t>(T), *positions = blank<int32_t>(T), *seen = blank<int32_t>((size_t)T * words);
        e = launch_attn_draft_tree(batch, T, words, parents, cu, cached, p[3], p[4], positions, seen, nullptr);
        fwrite(positions, 4, T, out);
        fwrite(seen, 4, (size_t)T * words, out);
    } else if (h[1] == 1) {  // accept
        const int log2_bs = p[2], max_blocks = p[3], capacity = p[4], gives_back = p[5];
        int32_t *tokens = array<int32_t>(T), *parents = array<int32_t>(T), *choices = array<int32_t>(T);
        int32_t *table = gives_back ? array<int32_t>((size_t)batch * max_blocks) : nullptr;
        int32_t *free_blocks = gives_back ? array<int32_t>(capacity) : nullptr, *n_free = gives_back ? array<int32_t>(1) : nullptr;
        int32_t *path = blank<int32_t>(T), *counts = blank<int32_t>(batch), *next = blank<int32_t>(batch), *lens = blank<int32_t>(batch), *left = blank<int32_t>(1);
        e = launch_attn_accept(batch, log2_bs, max_blocks, T, tokens, parents, choices, cu, cached, table, free_blocks, n_free, capacity,
                               path, counts, next, lens, left, nullptr);
        fwrite(path, 4, T, out);
        fwrite(counts, 4, batch, out);
        fwrite(next, 4, batch, out);
        fwrite(lens, 4, batch, out);
        fwrite(left, 4, 1, out);
        if (gives_back)
            fwrite(free_blocks, 4, capacity, out);
    } else {
        attn_shape_t s;
        s.n_q_heads = p[2], s.n_kv_heads = p[3], s.head_dim = p[4], s.block_size = p[5], s.io_dtype = p[6];
        const size_t esz = s.io_dtype == ATTN_DT_F32 ? 4 : 2;
        const int n_blocks = p[7], max_blocks = p[8];
        const size_t cache = (size_t)n_blocks * s.n_kv_heads * s.block_size * s.head_dim * esz;
        int32_t *table = array<int32_t>((size_t)batch * max_blocks);
        if (h[1] == 2) {  // keep
            const int n_caches = p[9];
            int32_t *path = array<int32_t>(T);
            std::vector<void *> caches;
            for (int c = 0; c < n_caches; ++c)
                caches.push_back(array<unsigned char>(cache));
            e = launch_attn_keep(s, batch, T, n_blocks, max_blocks, n_caches, caches.data(), table, cu, cached, path, nullptr);
            for (void *c : caches)
                fwrite(c, 1, cache, out);
        } else {  // attend
            const int window = p[9], sinks = p[10], max_new = p[11];
            float scale;
            memcpy(&scale, p + 12, 4);
            const size_t row = (size_t)s.n_q_heads * s.head_dim;
            AttnTrees trees;
            trees.words = p[13];
            trees.positions = array<int32_t>(T);
            trees.seen = array<int32_t>((size_t)T * trees.words);
            unsigned char *q = array<unsigned char>(T * row * esz), *k = array<unsigned char>(cache), *v = array<unsigned char>(cache);
            unsigned char *o = blank<unsigned char>(T * row * esz);
            float *lse = blank<float>((size_t)T * s.n_q_heads);
            const size_t need = attn_attend_tree_workspace(s, batch, T, max_new);
            unsigned char *ws = blank<unsigned char>(need);
            memset(ws, 0xFF, need);  // NaN patterns
            e = launch_attn_attend_tree(s, batch, T, n_blocks, max_blocks, q, row, k, v, table, cu, cached, scale, window, sinks, max_new, o, row,
                                   lse, ws, nullptr, trees);
            fwrite(o, 1, T * row * esz, out);
            fwrite(lse, 4, (size_t)T * s.n_q_heads, out);
        }
    }
    fclose(out);
    if (e != hipSuccess) {
        fprintf(stderr, "launch failed: %d\n", e);
        return 4;
    }
    return 0;
}
