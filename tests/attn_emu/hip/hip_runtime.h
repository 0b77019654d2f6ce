// What the attention kernels use beyond the stand-in of kernel_emu (test infrastructure only): lane exchanges of integers,
// ballots and the 16x16x32 product of fp16.  The product publishes every lane's operands between two lockstep points of the
// wave: the lanes of a wave run one after another between such points, and no other wave runs meanwhile.
#pragma once
#include "../../kernel_emu/hip/hip_runtime.h"

#include <map>
#include <vector>

namespace emu {
inline int bpermute(int addr, int v, int line) { return shfl(v, (addr >> 2) & 63, line); }
inline uint64_t ballot(bool v, int line)
{
    static bool said[64];
    const int l = thread_idx().x & 63;
    said[l] = v;
    wave_sync(line);
    uint64_t m = 0;
    for (int i = 0; i < 64; ++i)
        m |= (uint64_t)said[i] << i;
    wave_sync(line);
    return m;
}
inline f32x4 mfma_16x16x32_f16(f16x8 a, f16x8 b, f32x4 c, int line)
{
    // A: lane l holds row l%16, k = 8(l/16)+e.  B: column l%16, same k.  C/D: column l%16, row 4(l/16) + r.
    static float A[16][32], B[32][16];
    const int l = thread_idx().x & 63;
    for (int e = 0; e < 8; ++e) {
        A[l % 16][8 * (l / 16) + e] = (float)a[e];
        B[8 * (l / 16) + e][l % 16] = (float)b[e];
    }
    wave_sync(line);
    f32x4 d;
    for (int r = 0; r < 4; ++r) {
        double acc = (double)c[r];
        for (int k = 0; k < 32; ++k)
            acc += (double)A[4 * (l / 16) + r][k] * (double)B[k][l % 16];
        d[r] = (float)acc;
    }
    wave_sync(line);
    return d;
}
// Copies of 16 bytes per lane from memory into LDS, at once or when they are waited for; where to has to be the same in all lanes.
struct Copy {
    const void *from;
    unsigned char *to;
};
inline std::vector<Copy> &copies()  // of the lane that asks
{
    static std::map<unsigned, std::vector<Copy>> of;
    return of[thread_idx().x];
}
inline void copy16_to_lds(const void *from, uint32_t at, int line)
{
    if ((uint32_t)readfirstlane((int)at, line) != at)
        abort();
    unsigned char *to = lds_base() + at + 16 * (thread_idx().x & 63);
    memcpy(to, from, 16);
    if (env_int("EMU_LATE_COPIES")) {
        memset(to, 0xFF, 16);
        copies().push_back({from, to});
    }
}
inline void memory_wait(int line)
{
    wave_sync(line);
    for (const Copy &c : copies())
        memcpy(c.to, c.from, 16);
    copies().clear();
    wave_sync(line);
}
}  // namespace emu

#define __builtin_amdgcn_ds_bpermute(addr, v) emu::bpermute((addr), (v), __LINE__)
#define __builtin_amdgcn_sched_group_barrier(mask, n, id) ((void)0)
#define __ballot(v) emu::ballot((v), __LINE__)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) emu::mfma_16x16x32_f16((a), (b), (c), __LINE__)
