// Driver of the CPU emulation for the gated recurrence (test infrastructure only); the manner is emu_attn_main.cpp's.
//   emu_rec_main <in.bin> <out.bin> [order] [end|start]
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>

#include "rec_common.h"
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
    memset(p, 0x7E, n * sizeof(T));  // what no result is: every output must be written, and rows of no sequence must not
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
    rec_shape_t s;
    s.channels = p[0], s.io_dtype = p[1];
    memcpy(&s.sharpness, p + 2, 4);
    const int batch = p[3], T = p[4], C = s.channels, gap = p[5];  // gap: elements between rows beyond the channels
    const size_t esz = s.io_dtype == REC_DT_F32 ? 4 : 2, row = C + gap, n = T ? (T - 1) * row + C : 0, states = (size_t)batch * C;
    int32_t *cu = array<int32_t>(batch + 1);
    RecIo in;
    in.x = array<unsigned char>(n * esz), in.r = array<unsigned char>(n * esz), in.i = array<unsigned char>(n * esz);
    in.x_stride = in.r_stride = in.i_stride = row;
    float *decay = array<float>(C);
    if (h[1] == 0) {  // scan
        const int has_init = p[6], n_ckpt = p[7], save = p[8];
        RecScan a = {};
        a.in = in, a.decay = decay, a.cu = cu, a.T = T, a.batch = batch, a.n_ckpt = n_ckpt;
        a.init = has_init ? array<float>(states) : nullptr;
        a.ckpt = array<int32_t>(n_ckpt);
        a.y = blank<unsigned char>((size_t)T * C * esz), a.y_stride = C;
        a.final_states = blank<float>(states), a.ckpt_states = blank<float>((size_t)n_ckpt * C);
        const size_t rows = (T + REC_SAVED_EVERY - 1) / REC_SAVED_EVERY;
        a.saved = save ? blank<float>(rows * C) : nullptr;
        void *ws = blank<unsigned char>(rec_scan_workspace(s, batch, T, 0));
        e = launch_rec_scan(s, a, ws, nullptr);
        fwrite(a.y, esz, (size_t)T * C, out);
        fwrite(a.final_states, 4, states, out);
        fwrite(a.ckpt_states, 4, (size_t)n_ckpt * C, out);
        if (save)
            fwrite(a.saved, 4, rows * C, out);
    } else if (h[1] == 1) {  // gradients
        const int has_init = p[6], has_dy = p[7], has_final = p[8], wants_init = p[9];
        RecGrads a = {};
        a.in = in, a.decay = decay, a.cu = cu, a.T = T, a.batch = batch;
        a.init = has_init ? array<float>(states) : nullptr;
        a.dy = has_dy ? array<unsigned char>((size_t)T * C * esz) : nullptr, a.dy_stride = C;
        a.d_final = has_final ? array<float>(states) : nullptr;
        a.dx = blank<unsigned char>((size_t)T * C * esz), a.dr = blank<unsigned char>((size_t)T * C * esz), a.di = blank<unsigned char>((size_t)T * C * esz);
        a.d_decay = blank<float>(C), a.d_init = wants_init ? blank<float>(states) : nullptr;
        void *ws = blank<unsigned char>(rec_scan_workspace(s, batch, T, 2));
        e = launch_rec_grads(s, a, ws, nullptr);
        for (void *d : {a.dx, a.dr, a.di})
            fwrite(d, esz, (size_t)T * C, out);
        fwrite(a.d_decay, 4, C, out);
        if (wants_init)
            fwrite(a.d_init, 4, states, out);
    } else if (h[1] == 2) {  // step
        float *st = array<float>(states);
        unsigned char *y = blank<unsigned char>((size_t)T * C * esz);
        e = launch_rec_step(s, batch, in, decay, st, y, C, nullptr);
        fwrite(y, esz, (size_t)T * C, out);
        fwrite(st, 4, states, out);
    } else {  // tree, and the state that is kept
        float *st = array<float>(states), *nodes = blank<float>((size_t)T * C);
        int32_t *parents = array<int32_t>(T), *path = array<int32_t>(T), *counts = array<int32_t>(batch);
        unsigned char *y = blank<unsigned char>((size_t)T * C * esz);
        e = launch_rec_step_tree(s, batch, T, in, decay, st, cu, parents, y, C, nodes, nullptr);
        fwrite(y, esz, (size_t)T * C, out);
        fwrite(nodes, 4, (size_t)T * C, out);
        if (e == hipSuccess)
            e = launch_rec_keep(C, batch, T, st, nodes, cu, path, counts, nullptr);
        fwrite(st, 4, states, out);
    }
    fclose(out);
    if (e != hipSuccess) {
        fprintf(stderr, "launch failed: %d\n", e);
        return 4;
    }
    return 0;
}
