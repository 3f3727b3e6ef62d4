// Sampling of tokens: what the kernel and its entry point share.
#pragma once

#include "common.hpp"

namespace quarot {

constexpr int SAMPLE_MAX_VOCAB = 1 << 20;

struct SampleArgs {
    const void *logits;  // [rows, V], `stride` elements apart, binary16 or binary32
    int64_t stride;
    const float *u, *temperature, *top_p, *min_p;  // [rows] or null (u is always there)
    const int32_t *top_k;
    int32_t *tokens;
    int V;
    int log2_one;  // a weight of 1 is 2^log2_one
};

hipError_t launch_sample(const SampleArgs &a, bool f32, int64_t rows, hipStream_t s);

}  // namespace quarot
