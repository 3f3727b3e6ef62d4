// C ABI of the sampling: argument validation and launch.
#include "capi_util.hpp"
#include "sample.hpp"

#include <algorithm>

using namespace quarot;

extern "C" {

quarot_status quarot_sample(const void *logits, int64_t stride, int f32, const float *u,
                            const float *temperature, const int32_t *top_k, const float *top_p,
                            const float *min_p, int32_t *tokens, int64_t rows, int64_t vocab,
                            void *stream)
{
    if (rows < 0 || vocab <= 0 || (rows > 1 && stride < vocab))
        return QUAROT_ERR_INVALID_ARG;
    if (vocab > SAMPLE_MAX_VOCAB || rows > 0x3FFFFF || stride > (int64_t(1) << 32))
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if (rows == 0)
        return QUAROT_OK;
    if (!logits || !u || !tokens)
        return QUAROT_ERR_INVALID_ARG;
    for (const void *p : {static_cast<const void *>(u), static_cast<const void *>(temperature),
                          static_cast<const void *>(top_k), static_cast<const void *>(top_p),
                          static_cast<const void *>(min_p), static_cast<const void *>(tokens)})
        if (reinterpret_cast<uintptr_t>(p) & 3u)
            return QUAROT_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(logits) & (f32 ? 3u : 1u))
        return QUAROT_ERR_ALIGNMENT;
    quarot_status st = check_device(__func__);
    if (st)
        return st;
    SampleArgs a{};
    a.logits = logits;
    a.stride = stride;
    a.u = u;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.tokens = tokens;
    a.V = (int)vocab;
    // weights of a vocabulary sum up to less than 2^63, and a weight is exact in binary64
    int bits = 0;
    while ((int64_t(1) << bits) < vocab)
        ++bits;
    a.log2_one = std::min(62 - bits, 51);
    hipError_t e = launch_sample(a, f32 != 0, rows, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

}  // extern "C"
