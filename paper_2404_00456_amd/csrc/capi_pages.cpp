// C ABI of the cache's pages: argument validation and launches.
#include "capi_paged_util.hpp"
#include "pages.hpp"

using namespace quarot;

namespace {

quarot_status check_table(int64_t batch, int64_t max_pages, int64_t n_pages)
{
    if (batch <= 0 || max_pages <= 0 || n_pages <= 0)
        return QUAROT_ERR_INVALID_ARG;
    // (a table's positions, with pages of 16 tokens at least)
    if (batch > PAGES_MAX_BATCH || max_pages > kMaxTokens / 16 || n_pages > kMaxTokens)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    return QUAROT_OK;
}

template <class... P>
quarot_status check_ints(P... p)
{
    for (const void *x : {static_cast<const void *>(p)...}) {
        if (!x)
            return QUAROT_ERR_INVALID_ARG;
    }
    for (const void *x : {static_cast<const void *>(p)...}) {
        if (!aligned4(x))
            return QUAROT_ERR_ALIGNMENT;
    }
    return QUAROT_OK;
}

quarot_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (!ws || have < need)
        return QUAROT_ERR_WORKSPACE;
    return aligned16(ws) ? QUAROT_OK : QUAROT_ERR_ALIGNMENT;
}

void fill(PagesArgs &a, int32_t *table, int32_t *lens, int32_t *refs, int64_t B, int64_t P, int64_t n)
{
    a.table = table;
    a.lens = lens;
    a.refs = refs;
    a.B = (int)B;
    a.P = (int)P;
    a.n = (int)n;
}

}  // namespace

extern "C" {

size_t quarot_kv_pages_workspace_size(int64_t n_pages)
{
    return n_pages > 0 && n_pages <= kMaxTokens ? (size_t)n_pages * 4 * sizeof(int32_t) : 0;
}

quarot_status quarot_kv_pages_fork(int32_t *page_table, int32_t *seq_lens, int32_t *page_refs,
                                   const int32_t *parent, int64_t batch, int64_t max_pages,
                                   int64_t n_pages, void *stream)
{
    quarot_status st = check_table(batch, max_pages, n_pages);
    if (st || (st = check_ints(page_table, seq_lens, page_refs, parent)) || (st = check_device(__func__)))
        return st;
    ForkArgs a{};
    fill(a, page_table, seq_lens, page_refs, batch, max_pages, n_pages);
    a.parent = parent;
    hipError_t e = launch_pages_fork(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

quarot_status quarot_kv_pages_reserve(int32_t *page_table, int32_t *seq_lens, int32_t *page_refs,
                                      const int32_t *n_new, int32_t *cu_new, int32_t *copy_src,
                                      int32_t *copy_dst, int32_t *missing, int64_t batch,
                                      int64_t max_pages, int64_t n_pages, int64_t page_size,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    quarot_status st = check_table(batch, max_pages, n_pages);
    if (st)
        return st;
    if (page_size <= 0)
        return QUAROT_ERR_INVALID_ARG;
    if (page_size % 16 || page_size > kMaxTokens || max_pages > kMaxTokens / page_size)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if ((st = check_ints(page_table, seq_lens, page_refs, n_new, cu_new, copy_src, copy_dst, missing)) ||
        (st = check_workspace(workspace, workspace_bytes, quarot_kv_pages_workspace_size(n_pages))) ||
        (st = check_device(__func__)))
        return st;
    ReserveArgs a{};
    fill(a, page_table, seq_lens, page_refs, batch, max_pages, n_pages);
    a.n_new = n_new;
    a.cu = cu_new;
    a.src = copy_src;
    a.dst = copy_dst;
    a.missing = missing;
    a.ws = static_cast<int32_t *>(workspace);
    a.page = (int)page_size;
    a.div = paged::divisor(a.page);
    hipError_t e = launch_pages_reserve(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

quarot_status quarot_kv_pages_compact(int32_t *page_table, int32_t *page_refs, int32_t *move_src,
                                      int32_t *move_dst, int32_t *n_live, int64_t batch,
                                      int64_t max_pages, int64_t n_pages, void *workspace,
                                      size_t workspace_bytes, void *stream)
{
    quarot_status st = check_table(batch, max_pages, n_pages);
    if (st)
        return st;
    if ((st = check_ints(page_table, page_refs, n_live)) ||
        (n_pages > 1 && (st = check_ints(move_src, move_dst))) ||
        (st = check_workspace(workspace, workspace_bytes, quarot_kv_pages_workspace_size(n_pages))) ||
        (st = check_device(__func__)))
        return st;
    CompactArgs a{};
    fill(a, page_table, nullptr, page_refs, batch, max_pages, n_pages);
    a.src = move_src;
    a.dst = move_dst;
    a.live = n_live;
    a.ws = static_cast<int32_t *>(workspace);
    hipError_t e = launch_pages_compact(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

quarot_status quarot_kv_pages_copy(const quarot_paged_kv *cache, const int32_t *src, const int32_t *dst,
                                   int64_t count, void *stream)
{
    if (!cache || count < 0 || cache->n_kv_heads <= 0 || cache->head_dim <= 0 || cache->group <= 0 ||
        cache->n_pages <= 0 || cache->page_size <= 0)
        return QUAROT_ERR_INVALID_ARG;
    if (!head_dim_ok(cache->head_dim) || !group_ok(cache->group, cache->head_dim) || cache->page_size % 16 ||
        cache->page_size > kMaxTokens || cache->n_pages > 0x7FFFFFFF || cache->n_kv_heads > 0xFFFF ||
        count > kMaxTokens)
        return QUAROT_ERR_UNSUPPORTED_SIZE;
    if (count == 0)
        return QUAROT_OK;
    quarot_status st = check_ints(src, dst);
    if (st)
        return st;
    if (!cache->k_codes || !cache->k_scale || !cache->k_zero || !cache->v_codes || !cache->v_scale ||
        !cache->v_zero)
        return QUAROT_ERR_INVALID_ARG;
    if (!aligned16(cache->k_codes) || !aligned16(cache->k_scale) || !aligned16(cache->k_zero) ||
        !aligned16(cache->v_codes) || !aligned16(cache->v_scale) || !aligned16(cache->v_zero))
        return QUAROT_ERR_ALIGNMENT;
    if ((st = check_device(__func__)))
        return st;
    CopyArgs a{};
    a.kp = PagedPool{cache->k_codes, cache->k_scale, cache->k_zero};
    a.vp = PagedPool{cache->v_codes, cache->v_scale, cache->v_zero};
    a.src = src;
    a.dst = dst;
    a.count = (int)count;
    a.n = (int)cache->n_pages;
    const int64_t rows = cache->n_kv_heads * cache->page_size;
    a.code_bytes = rows * (cache->head_dim / 2);
    a.const_bytes = rows * (cache->head_dim / cache->group) * 2;
    hipError_t e = launch_pages_copy(a, (hipStream_t)stream);
    return e == hipSuccess ? QUAROT_OK : hip_fail(e);
}

}  // extern "C"
