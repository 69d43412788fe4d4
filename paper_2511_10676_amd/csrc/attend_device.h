// What the attention kernels over 16- or 32-bit and over 4-bit caches share: exponentials of differences of scores.
#pragma once

#include "cache_device.h"

namespace paep {

static constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;

// Of differences of scores only: a score in units of log2 may be past the largest number where the score itself is not.
__device__ __forceinline__ float exp_(float v) { return __builtin_amdgcn_exp2f(v * LOG2E); }
// the reference point of exponentials whose maximum is m: 0 where nothing was above -infinity
__device__ __forceinline__ float origin(float m) { return m == -__builtin_inff() ? 0.0f : m; }

}  // namespace paep
