// C ABI of the rotary positions and the paged KV cache: argument validation and
// launches.  Every check runs on the host before any device work.
#include "capi_util.hpp"
#include "paged.hpp"

using namespace quarot;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 30;  // positions of a table, and T * heads

constexpr int64_t kMaxStride = int64_t(1) << 32;

bool aligned4(const void *p)
{
    return (reinterpret_cast<uintptr_t>(p) & 3u) == 0;
}

bool head_dim_ok(int64_t d)
{
    return d == 64 || d == 128 || d == 256;
}

bool group_ok(int64_t group, int64_t d)
{
    return group >= 32 && group <= d && !(group & (group - 1));
}

quarot_status check_stride(int64_t stride, int64_t heads, int64_t D)
{
    if (stride < heads * D)
        return QUAROT_ERR_INVALID_ARG;
    if (stride > kMaxStride)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    return stride % 8 ? QUAROT_ERR_ALIGNMENT : QUAROT_OK;
}

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

quarot_status check_cache_sizes(const quarot_paged_kv *c, int64_t T)
{
    if (!c || T < 0 || c->batch <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->group <= 0 ||
        c->n_pages <= 0 || c->page_size <= 0 || c->max_pages <= 0)
        return QUAROT_ERR_INVALID_ARG;
    if (!head_dim_ok(c->head_dim) || !group_ok(c->group, c->head_dim) || c->page_size % 16 || c->page_size > kMaxTokens ||
        c->max_pages > kMaxTokens / c->page_size || c->n_pages > 0x7FFFFFFF ||
        c->n_kv_heads > 0xFFFF || c->batch > 0xFFFFFF || T > kMaxTokens)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    return QUAROT_OK;
}

quarot_status check_cache_pointers(const quarot_paged_kv *c)
{
    if (!c->k_codes || !c->k_scale || !c->k_zero || !c->v_codes || !c->v_scale || !c->v_zero ||
        !c->page_table || !c->seq_lens || !c->cu_new)
        return QUAROT_ERR_INVALID_ARG;
    if (!aligned16(c->k_codes) || !aligned16(c->k_scale) || !aligned16(c->k_zero) ||
        !aligned16(c->v_codes) || !aligned16(c->v_scale) || !aligned16(c->v_zero) ||
        !aligned4(c->page_table) || !aligned4(c->seq_lens) || !aligned4(c->cu_new))
        return QUAROT_ERR_ALIGNMENT;
    return QUAROT_OK;
}

void fill_cache(const quarot_paged_kv *c, int64_t T, PagedPool &k, PagedPool &v, PagedMap &m)
{
    k = PagedPool{c->k_codes, c->k_scale, c->k_zero};
    v = PagedPool{c->v_codes, c->v_scale, c->v_zero};
    m.table = c->page_table;
    m.len = c->seq_lens;
    m.cu = c->cu_new;
    m.T = (int)T;
    m.B = (int)c->batch;
    m.max_pages = (int)c->max_pages;
    m.n_pages = (int)c->n_pages;
    m.page = (int)c->page_size;
    m.div = paged::divisor(m.page);
}

// A launch holds fewer than 2^32 threads.
bool plan_fits(const paged::Plan &p, int64_t T, int64_t batch, int64_t hkv, int64_t rep)
{
    for (int i = 0; i < p.n; ++i)
        if (paged::slots(p.part[i], T, batch, rep) * hkv * p.part[i].splits >
            0xFFFFFFFFll / paged::MAX_THREADS)
            return false;
    return true;
}

// The launches of a plan use the workspace one after the other.
size_t attention_workspace(const paged::Plan &p, int64_t T, int64_t batch, int64_t hkv, int64_t rep,
                           int64_t head_dim)
{
    size_t need = 0;
    for (int i = 0; i < p.n; ++i)
        need = std::max(need, (size_t)(paged::part_rows(p.part[i], T, batch, rep) * hkv * p.part[i].splits) *
                                  (size_t)(head_dim + 2) * sizeof(float));
    return need;
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
    quarot_status st = check_cache_sizes(cache, T);
    if (st)
        return st;
    if (n_heads <= 0 || n_heads % cache->n_kv_heads || max_seq_len <= 0 || window < 0 ||
        n_sinks < 0 || !(sm_scale > 0.0f) || !std::isfinite(sm_scale))
        return QUAROT_ERR_INVALID_ARG;
    if (n_heads > 0xFFFF || T * n_heads > kMaxTokens)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if (T == 0)
        return QUAROT_OK;
    if (!q || !out)
        return QUAROT_ERR_INVALID_ARG;
    if ((st = check_cache_pointers(cache)))
        return st;
    const int64_t D = cache->head_dim;
    if ((st = check_stride(q_stride, n_heads, D)) || (st = check_stride(out_stride, n_heads, D)))
        return st;
    if (!aligned16(q) || !aligned16(out))
        return QUAROT_ERR_ALIGNMENT;
    window = std::min(window, kMaxTokens);
    n_sinks = std::min(n_sinks, kMaxTokens);
    const int64_t hkv = cache->n_kv_heads, rep = n_heads / hkv;
    const paged::Plan p = paged::plan(T, cache->batch, hkv, rep, D,
                                      std::min(max_seq_len, kMaxTokens), window, n_sinks);
    if (!plan_fits(p, T, cache->batch, hkv, rep))
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    const size_t need = attention_workspace(p, T, cache->batch, hkv, rep, D);
    if (need && (!workspace || workspace_bytes < need))
        return QUAROT_ERR_WORKSPACE;
    if (need && !aligned16(workspace))
        return QUAROT_ERR_ALIGNMENT;
    if ((st = check_device(__func__)))
        return st;
    PagedAttnArgs a{};
    a.q = q;
    a.q_stride = q_stride;
    a.out = out;
    a.out_stride = out_stride;
    fill_cache(cache, T, a.kp, a.vp, a.map);
    a.hq = (int)n_heads;
    a.hkv = (int)hkv;
    a.rep = (int)rep;
    a.D = (int)D;
    a.G = (int)cache->group;
    a.window = (int)window;
    a.sinks = (int)n_sinks;
    a.sm_scale = sm_scale;
    hipError_t e = hipSuccess;
    for (int i = 0; i < p.n && e == hipSuccess; ++i) {
        const paged::Part &part = p.part[i];
        a.which = part.which;
        a.splits = part.splits;
        a.least = part.least;
        a.part_o = static_cast<float *>(workspace);
        a.part_ml = a.part_o + (size_t)(paged::part_rows(part, T, cache->batch, rep) * hkv * part.splits * D);
        e = launch_paged_attention(a, part.rows, (hipStream_t)stream);
    }
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

}  // extern "C"
