// C ABI of the rotary positions and the paged KV cache: argument validation and
// launches.  Every check runs on the host before any device work.
#include "capi_paged_util.hpp"

using namespace quarot;

namespace {

// Sizes of the rotary positions; fills `ro`.
quarot_status check_rotary(const quarot_rotary *r, int64_t T, int64_t D, bool own_positions,
                           RopeArgs &ro)
{
    ro = RopeArgs{};
    if (!r || !r->inv_freq)
        return own_positions ? QUAROT_OK : QUAROT_ERR_INVALID_ARG;
    if (r->n_axes < 1 || r->rot_dim <= 0)
        return QUAROT_ERR_INVALID_ARG;
    if (r->n_axes > 4 || r->rot_dim % 16 || r->rot_dim > D || r->pos_stride > kMaxStride)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if (r->positions ? r->pos_stride < T : T > 0 && (!own_positions || r->n_axes != 1))
        return QUAROT_ERR_INVALID_ARG;
    if (!aligned4(r->positions) || !aligned4(r->inv_freq))
        return QUAROT_ERR_ALIGNMENT;
    ro.pos = r->positions;
    ro.pos_stride = r->pos_stride;
    ro.inv_freq = r->inv_freq;
    ro.half = r->rot_dim / 2;
    ro.interleaved = r->interleaved != 0;
    for (int f = 0; r->axis_map && f < ro.half; ++f) {
        if (r->axis_map[f] >= r->n_axes)
            return QUAROT_ERR_INVALID_ARG;
        ro.axis[f >> 4] |= (uint32_t)r->axis_map[f] << (2 * (f & 15));
    }
    return QUAROT_OK;
}

}  // namespace

extern "C" {

quarot_status quarot_rope(const quarot_f16 *x, int64_t x_stride, quarot_f16 *y, int64_t y_stride,
                          const quarot_rotary *rotary, int64_t T, int64_t n_heads,
                          int64_t head_dim, int rotate, void *stream)
{
    if (T < 0 || n_heads <= 0 || head_dim <= 0)
        return QUAROT_ERR_INVALID_ARG;
    if (!head_dim_ok(head_dim) || n_heads > 0xFFFF || T > 0x7FFFFFFF / APPEND_THREADS)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    AppendArgs a{};
    quarot_status st = check_rotary(rotary, T, head_dim, false, a.rope);
    if (st)
        return st;
    if (T == 0)
        return QUAROT_OK;
    if (!x || !y)
        return QUAROT_ERR_INVALID_ARG;
    if ((st = check_stride(x_stride, n_heads, head_dim)) ||
        (st = check_stride(y_stride, n_heads, head_dim)))
        return st;
    if (x == y && x_stride != y_stride)
        return QUAROT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(y))
        return QUAROT_ERR_ALIGNMENT;
    if ((st = check_device(__func__)))
        return st;
    a.q = x;
    a.q_stride = x_stride;
    a.qo = y;
    a.qo_stride = y_stride;
    a.map.T = (int)T;
    a.hq = (int)n_heads;
    a.D = (int)head_dim;
    a.rot_k = rotate != 0;
    a.c = rotation_scale(head_dim);
    hipError_t e = launch_append(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

quarot_status quarot_kv_append_paged(const quarot_f16 *q, int64_t q_stride, quarot_f16 *q_out,
                                     int64_t q_out_stride, const quarot_f16 *k, int64_t k_stride,
                                     const quarot_f16 *v, int64_t v_stride,
                                     const quarot_paged_kv *cache, const quarot_rotary *rotary,
                                     int64_t T, int64_t n_heads, int rotate_k, int rotate_v,
                                     float clip_ratio, void *stream)
{
    quarot_status st = check_cache_sizes(cache, T);
    if (st)
        return st;
    if (n_heads < 0 || !clip_ok(clip_ratio))
        return QUAROT_ERR_INVALID_ARG;
    if (n_heads > 0xFFFF || T > 0x7FFFFFFF / APPEND_THREADS)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    AppendArgs a{};
    if ((st = check_rotary(rotary, T, cache->head_dim, true, a.rope)))
        return st;
    if (T == 0)
        return QUAROT_OK;
    const int64_t D = cache->head_dim;
    if (!k || !v || (n_heads > 0 && (!q || !q_out)) || (n_heads == 0 && (q || q_out)))
        return QUAROT_ERR_INVALID_ARG;
    if ((st = check_cache_pointers(cache)))
        return st;
    if ((st = check_stride(k_stride, cache->n_kv_heads, D)) ||
        (st = check_stride(v_stride, cache->n_kv_heads, D)))
        return st;
    if (n_heads > 0) {
        if ((st = check_stride(q_stride, n_heads, D)) || (st = check_stride(q_out_stride, n_heads, D)))
            return st;
        if (q == q_out && q_stride != q_out_stride)
            return QUAROT_ERR_INVALID_ARG;
    }
    if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(v))
        return QUAROT_ERR_ALIGNMENT;
    if ((st = check_device(__func__)))
        return st;
    a.q = q;
    a.q_stride = q_stride;
    a.qo = q_out;
    a.qo_stride = q_out_stride;
    a.k = k;
    a.k_stride = k_stride;
    a.v = v;
    a.v_stride = v_stride;
    fill_cache(cache, T, a.kp, a.vp, a.map);
    a.hq = (int)n_heads;
    a.hkv = (int)cache->n_kv_heads;
    a.D = (int)D;
    a.G = (int)cache->group;
    a.rot_k = rotate_k != 0;
    a.rot_v = rotate_v != 0;
    a.c = rotation_scale(D);
    a.clip = clip_ratio;
    hipError_t e = launch_append(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

size_t quarot_kv_paged_attention_workspace_size(int64_t T, int64_t batch, int64_t n_heads,
                                                int64_t n_kv_heads, int64_t head_dim,
                                                int64_t group, int64_t max_seq_len, int64_t window,
                                                int64_t n_sinks)
{
    if (T <= 0 || T > kMaxTokens || batch <= 0 || batch > 0xFFFFFF || n_heads <= 0 ||
        n_heads > 0xFFFF || T * n_heads > kMaxTokens || n_kv_heads <= 0 || n_heads % n_kv_heads ||
        !head_dim_ok(head_dim) || !group_ok(group, head_dim) || max_seq_len <= 0 || window < 0 ||
        n_sinks < 0)
        return 0;
    const int64_t rep = n_heads / n_kv_heads;
    const paged::Plan p = paged::plan(T, batch, n_kv_heads, rep, head_dim,
                                      std::min(max_seq_len, kMaxTokens), std::min(window, kMaxTokens),
                                      std::min(n_sinks, kMaxTokens));
    return plan_fits(p, T, batch, n_kv_heads, rep)
               ? attention_workspace(p, T, batch, n_kv_heads, rep, head_dim)
               : 0;
}

quarot_status quarot_kv_paged_attention(const quarot_f16 *q, int64_t q_stride, quarot_f16 *out,
                                        int64_t out_stride, const quarot_paged_kv *cache, int64_t T,
                                        int64_t n_heads, int64_t max_seq_len, int64_t window,
                                        int64_t n_sinks, float sm_scale, void *workspace,
                                        size_t workspace_bytes, void *stream)
{
    return paged_attention_call(__func__, PagedAttnArgs{}, launch_paged_attention, q, q_stride, out, out_stride,
                                cache, T, n_heads, max_seq_len, window, n_sinks, sm_scale, workspace,
                                workspace_bytes, stream);
}

}  // extern "C"
