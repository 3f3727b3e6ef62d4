// Scored attention over the paged 4-bit KV cache with caps far above the scores.
#include "paged_kernels.hpp"

namespace quarot {

hipError_t launch_large_cap_attention(const ScoredAttnArgs &a, int rows, hipStream_t s)
{
    return a.slopes ? go_dims<Scored<LARGE_CAP, true>>(a, rows, s) : go_dims<Scored<LARGE_CAP, false>>(a, rows, s);
}

}  // namespace quarot
