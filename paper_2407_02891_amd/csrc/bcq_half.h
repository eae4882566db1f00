// The two 16-bit element types of the serving operators (not public): conversions and matrix instructions by type.
#pragma once
#include "bcq_device.h"

namespace bcq {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 h16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

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

// Two values rounded to nearest even in one instruction; the first in the low half.
template <bool BF>
__device__ __forceinline__ uint32_t from_float2(float a, float b)
{
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), b16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), h16x2));
}

// The same, rounded toward zero.
template <bool BF>
__device__ __forceinline__ uint32_t toward_zero2(float a, float b)
{
    if constexpr (BF) return __builtin_bit_cast(uint32_t, a) >> 16 | (__builtin_bit_cast(uint32_t, b) & 0xffff0000u);
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

template <bool BF>
__device__ __forceinline__ f32x2 to_float2(uint32_t pair)
{
    if constexpr (BF) return f32x2{__builtin_bit_cast(float, pair << 16), __builtin_bit_cast(float, pair & 0xffff0000u)};
    else return f32x2{half_bits_to_float(pair & 0xffffu), half_bits_to_float(pair >> 16)};
}

// sum + 0 * the pair's elements: NaN once one of them was an infinity or a NaN.
template <bool BF>
__device__ __forceinline__ float times_zero(uint32_t pair, float sum)
{
    if constexpr (BF) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b16x2, pair), b16x2{0, 0}, sum, false);
    else return __builtin_amdgcn_fdot2(__builtin_bit_cast(h16x2, pair), h16x2{0, 0}, sum, false);
}

template <bool BF>
constexpr uint32_t kOne = BF ? 0x3f80u : 0x3c00u;

// One in the place of an infinity of the given sign bit and of a NaN, zero elsewhere.
template <bool BF>
__device__ __forceinline__ uint32_t ones_where_infinite(uint32_t pair, uint32_t sign)
{
    constexpr uint32_t kExponent = BF ? 0x7f80u : 0x7c00u;
    const auto one = [&](uint32_t h) { return (h & 0x7fffu) > kExponent || h == (kExponent | sign) ? kOne<BF> : 0u; };
    return one(pair & 0xffffu) | one(pair >> 16) << 16;
}

// Zero in the place of infinities and NaN.
template <bool BF>
__device__ __forceinline__ uint32_t finite_only(uint32_t pair)
{
    constexpr uint32_t kExponent = BF ? 0x7f80u : 0x7c00u;
    return ((pair & kExponent) == kExponent ? 0u : pair & 0xffffu) | ((pair >> 16 & kExponent) == kExponent ? 0u : pair & 0xffff0000u);
}

// D[i][j] = C[i][j] + sum_k A[i][k] B[k][j].  16 x 16 x 32: lane 16 g + r holds A[r][8 g ..] and B[8 g ..][r], and of C and D
// rows 4 g .. 4 g + 3 of column r.  The 32 k's may be numbered in any way that A and B share.
template <bool BF>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
}

// 32 x 32 x 16: lane 32 g + r holds A[r][8 g ..] and B[8 g ..][r], and of C and D rows 8 q + 4 g + i of column r in element 4 q + i.
template <bool BF>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
}

// Sixteen lanes give the places of four rows of sixteen 16-bit elements in LDS (lane a: row a / 4, elements 4 (a mod 4) ..) and
// get a column each: lane a element a of the four rows.
__device__ __forceinline__ u32x2 lds_column(const uint16_t *row_part)
{
    typedef __attribute__((address_space(3))) s16x4 *lds_ptr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(row_part)));
}

// Sum and maximum over the four lanes 16 apart / the two lanes 32 apart; every lane gets the result.
__device__ __forceinline__ float max_over_groups(float v)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
    a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
}
__device__ __forceinline__ float sum_over_groups(float v)
{
    auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
    a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
}

}  // namespace bcq
