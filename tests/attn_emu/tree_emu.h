// What the attention of trees uses beyond the stand-in of the other attention kernels (test infrastructure only): a wait for all copies
// into LDS but the last few.
#pragma once
#include <hip/hip_runtime.h>

namespace emu {
inline void memory_wait_but(size_t n, int line)
{
    wave_sync(line);
    std::vector<Copy> &c = copies();
    const size_t done = c.size() > n ? c.size() - n : 0;
    for (size_t i = 0; i < done; ++i)
        memcpy(c[i].to, c[i].from, 16);
    c.erase(c.begin(), c.begin() + done);
    wave_sync(line);
}
}  // namespace emu
