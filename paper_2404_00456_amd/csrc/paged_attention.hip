// Attention over the paged 4-bit KV cache: causal, with a sliding window and sinks.
#include "paged_kernels.hpp"

namespace quarot {

hipError_t launch_paged_attention(const PagedAttnArgs &a, int rows, hipStream_t s)
{
    return go_dims<Plain>(a, rows, s);
}

}  // namespace quarot
