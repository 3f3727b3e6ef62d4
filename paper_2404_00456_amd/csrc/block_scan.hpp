// Sums over the threads of a block, in order.
#pragma once

#include "common.hpp"

namespace quarot {

// v of the lane that a DPP pattern names, 0 where it names none.
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T lane_before(T v)
{
    auto half = [](uint32_t x) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
    };
    if constexpr (sizeof(T) == 8)
        return (T)((uint64_t)half((uint32_t)((uint64_t)v >> 32)) << 32 | half((uint32_t)v));
    else
        return (T)half((uint32_t)v);
}

// The sum of v over the lanes up to this one: within rows of 16, then from row to row.
template <class T>
__device__ __forceinline__ T wave_scan(T v)
{
    v += lane_before<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
    v += lane_before<0x112, 0xF>(v);
    v += lane_before<0x114, 0xF>(v);
    v += lane_before<0x118, 0xF>(v);
    v += lane_before<0x142, 0xA>(v);  // the last lane of rows 0 and 2 to rows 1 and 3
    v += lane_before<0x143, 0xC>(v);  // that of the first half to the second
    return v;
}

template <class T>
__device__ __forceinline__ T lane_value(T v, int lane)
{
    const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
    if constexpr (sizeof(T) == 8)
        return (T)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)v >> 32), lane) << 32 | lo);
    else
        return (T)lo;
}

// The largest v >= 0 of a wave.
__device__ __forceinline__ int wave_max(int v)
{
    v = max(v, lane_before<0x111, 0xF>(v));
    v = max(v, lane_before<0x112, 0xF>(v));
    v = max(v, lane_before<0x114, 0xF>(v));
    v = max(v, lane_before<0x118, 0xF>(v));
    v = max(v, lane_before<0x142, 0xA>(v));
    v = max(v, lane_before<0x143, 0xC>(v));
    return __builtin_amdgcn_readlane(v, 63);
}

// The sum of v over the threads before this one; `all` the sum of all.  `sums` holds one
// value a wave (16 at most); every thread of the block calls it.  (By shuffles and a loop
// over the waves' sums it took half a microsecond in 64 bits.)
template <int WAVES, class T>
__device__ __forceinline__ T block_scan(T v, T *sums, T &all)
{
    static_assert(WAVES <= 16, "a row of lanes");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T x = wave_scan(v);
    __syncthreads();  // (the last scan's sums are read)
    if (lane == 63)
        sums[wave] = x;
    __syncthreads();
    const T s = wave_scan(lane < WAVES ? sums[lane & (WAVES - 1)] : (T)0);
    all = lane_value(s, WAVES - 1);
    return (wave ? lane_value(s, wave - 1) : (T)0) + x - v;
}

}  // namespace quarot
