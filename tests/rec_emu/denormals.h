// rec_emu's stand-in with exp2, reciprocal and roots as gfx950's instructions compute them (test infrastructure only): a denormal
// operand counts as 0, and so does a result that would be one, although sums and products keep both.
#pragma once
#include "hip/hip_runtime.h"

namespace emu {
inline float flushed(float v) { return v > -0x1p-126f && v < 0x1p-126f ? copysignf(0.0f, v) : v; }
}  // namespace emu
#undef __builtin_amdgcn_exp2f
#undef __builtin_amdgcn_rcpf
#undef __builtin_amdgcn_sqrtf
#undef __builtin_amdgcn_rsqf
#define __builtin_amdgcn_exp2f(x) emu::flushed(exp2f(emu::flushed(x)))
#define __builtin_amdgcn_rcpf(x) emu::flushed(1.0f / emu::flushed(x))
#define __builtin_amdgcn_sqrtf(x) sqrtf(emu::flushed(x))
#define __builtin_amdgcn_rsqf(x) (1.0f / sqrtf(emu::flushed(x)))
