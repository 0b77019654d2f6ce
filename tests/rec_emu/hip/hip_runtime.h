// What the kernels of the gated recurrence use beyond the stand-in of attn_emu (test infrastructure only): roots, and atomics
// between workgroups, which run here one after another.
#pragma once
#include "../../attn_emu/hip/hip_runtime.h"

namespace emu {
template <typename T> inline T fetch_add(T *p, T v)
{
    const T old = *p;
    *p += v;
    return old;
}
}  // namespace emu
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_store(p, v, order, scope) ((void)(*(p) = (v)))
#define __hip_atomic_fetch_add(p, v, order, scope) emu::fetch_add((p), (v))
#define __builtin_amdgcn_sqrtf(x) sqrtf(x)
#define __builtin_amdgcn_rsqf(x) (1.0f / sqrtf(x))
static inline const char *hipGetErrorString(int) { return "error"; }
