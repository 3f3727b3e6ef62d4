// Sums over the threads of a block, in order.
#pragma once

#include "common.hpp"

namespace quarot {

// The sum of v over the threads before this one; `all` the sum of all.  `sums` holds one
// value a wave; every thread of the block calls it.
template <int WAVES, class T>
__device__ __forceinline__ T block_scan(T v, T *sums, T &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T x = v;
    for (int d = 1; d < 64; d <<= 1) {
        const T y = __shfl_up(x, d);
        x += lane >= d ? y : 0;
    }
    __syncthreads();  // (the last scan's sums are read)
    if (lane == 63)
        sums[wave] = x;
    __syncthreads();
    T before = 0;
    all = 0;
    for (int w = 0; w < WAVES; ++w) {
        const T s = sums[w];
        before += w < wave ? s : 0;
        all += s;
    }
    return before + x - v;
}

}  // namespace quarot
