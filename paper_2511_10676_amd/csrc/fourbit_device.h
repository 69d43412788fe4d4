// Numbers of 4 bits in device code: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, times a power of two that 32 neighbours share.
#pragma once

#include "paep_device.h"

namespace paep {

// What stands for the power 2^(byte - 127) where appended: with these every number of a group is 0 or a normal fp32 and bf16 number.
static constexpr int FOUR_LEAST_BYTE = 2, FOUR_MOST_BYTE = 252;

// both codes of byte B of a register as bf16 numbers, exactly (scale: a power of two, or infinite, its bits 255 << 23: NaN)
template <int B> __device__ __forceinline__ uint32_t pair_bf16(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

}  // namespace paep
