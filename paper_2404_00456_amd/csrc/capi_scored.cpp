// C ABI of the scored attention over the paged KV cache: argument validation and launches.
#include "capi_paged_util.hpp"

using namespace quarot;

extern "C" {

quarot_status quarot_kv_paged_attention_scored(const quarot_f16 *q, int64_t q_stride, quarot_f16 *out,
                                               int64_t out_stride, const quarot_paged_kv *cache,
                                               const quarot_scoring *scoring, int64_t T, int64_t n_heads,
                                               int64_t max_seq_len, int64_t window, int64_t n_sinks,
                                               float sm_scale, void *workspace, size_t workspace_bytes,
                                               void *stream)
{
    if (!scoring || !(scoring->cap >= 0.0f) || !std::isfinite(scoring->cap))
        return QUAROT_ERR_INVALID_ARG;
    // (exponents of the cap's tanh stay within binary32, and so does its reciprocal)
    if (scoring->cap > 0.0f && !(scoring->cap >= 0x1p-64f && scoring->cap <= 0x1p64f))
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if (!aligned4(scoring->slopes) || !aligned4(scoring->begin) || !aligned4(scoring->end))
        return QUAROT_ERR_ALIGNMENT;
    if (scoring->cap == 0.0f && !scoring->slopes && !scoring->begin && !scoring->end)
        return paged_attention_call(__func__, PagedAttnArgs{}, launch_paged_attention, q, q_stride, out,
                                    out_stride, cache, T, n_heads, max_seq_len, window, n_sinks, sm_scale,
                                    workspace, workspace_bytes, stream);
    ScoredAttnArgs a{};
    a.cap = scoring->cap;
    a.slopes = scoring->slopes;
    a.begin = scoring->begin;
    a.end = scoring->end;
    return paged_attention_call(__func__, a, launch_scored_attention, q, q_stride, out, out_stride, cache, T,
                                n_heads, max_seq_len, window, n_sinks, sm_scale, workspace,
                                workspace_bytes, stream);
}

}  // extern "C"
