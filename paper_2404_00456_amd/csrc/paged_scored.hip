// Scored attention over the paged 4-bit KV cache: spans of each query's own, scores capped
// by a tanh, slopes by distance.
#include "paged_kernels.hpp"

namespace quarot {

hipError_t launch_scored_attention(const ScoredAttnArgs &a, int rows, hipStream_t s)
{
    if (a.cap > CAP_LARGE)
        return launch_large_cap_attention(a, rows, s);
    if (a.cap > 0.0f)
        return a.slopes ? go_dims<Scored<CAP, true>>(a, rows, s) : go_dims<Scored<CAP, false>>(a, rows, s);
    return a.slopes ? go_dims<Scored<NO_CAP, true>>(a, rows, s) : go_dims<Scored<NO_CAP, false>>(a, rows, s);
}

}  // namespace quarot
