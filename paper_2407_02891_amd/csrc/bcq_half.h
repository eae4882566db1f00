// The two 16-bit element types of the serving operators (not public): conversions and matrix instructions by type.
#pragma once
#include "bcq_device.h"

namespace bcq {

// BF: bfloat16, else binary16.
template <bool BF>
__device__ __forceinline__ float to_float(uint32_t bits16)
{
    return BF ? __builtin_bit_cast(float, bits16 << 16) : half_bits_to_float(bits16 & 0xffffu);
}

// Round to nearest even.
template <bool BF>
__device__ __forceinline__ uint16_t from_float(float v)
{
    if constexpr (BF) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    else return float_to_half_bits(v);
}

}  // namespace bcq
