// Sums over the lanes of a wave (not public).
#pragma once
#include <hip/hip_runtime.h>

#include <stdint.h>

namespace bcq {

namespace {

__device__ __forceinline__ int from_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
template <int CTRL>
__device__ __forceinline__ int in_row(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }

// The same of 64 bits, by halves.
template <class T>
__device__ __forceinline__ T from_lane(T v, int lane)
{
    static_assert(sizeof(T) == 8, "");
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(T, (uint64_t)(uint32_t)from_lane((int)(b >> 32), lane) << 32 | (uint32_t)from_lane((int)b, lane));
}
template <int CTRL, class T>
__device__ __forceinline__ T in_row(T v)
{
    static_assert(sizeof(T) == 8, "");
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(T, (uint64_t)(uint32_t)in_row<CTRL>((int)(b >> 32)) << 32 | (uint32_t)in_row<CTRL>((int)b));
}

// Sum over the lanes up to and with this one: in rows of sixteen by shifts, then the rows before.
template <class T>
__device__ __forceinline__ T sum_upto(T v, int lane)
{
    v += in_row<0x111>(v);
    v += in_row<0x112>(v);
    v += in_row<0x114>(v);
    v += in_row<0x118>(v);
    const T r0 = from_lane(v, 15), r1 = r0 + from_lane(v, 31), r2 = r1 + from_lane(v, 47);
    return v + (lane < 32 ? lane < 16 ? T(0) : r0 : lane < 48 ? r1 : r2);
}
template <class T>
__device__ __forceinline__ T sum_all(T v)
{
    v += in_row<0x111>(v);
    v += in_row<0x112>(v);
    v += in_row<0x114>(v);
    v += in_row<0x118>(v);
    return from_lane(v, 15) + from_lane(v, 31) + (from_lane(v, 47) + from_lane(v, 63));
}

}  // namespace

}  // namespace bcq
