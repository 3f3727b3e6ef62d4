// The paged 4-bit KV cache: what its kernels and their launchers share.
//
// A batch holds the new tokens of B sequences one after the other: rows
// cu[b] .. cu[b + 1] - 1 of T belong to sequence b, whose cache holds len[b]
// tokens with the new ones, so new token i of n sits at position
// len - n + i.  Position t of sequence b is slot t % page of page
// table[b][t / page] of the pools.  All of cu, len and table live on the
// device: kernels bound what they read from them (a page outside the pool is
// no page, a row outside 0 .. T is no row), so that no content of theirs
// leads outside a buffer.
#pragma once

#include "common.hpp"
#include "paged_plan.hpp"

namespace quarot {

constexpr int APPEND_THREADS = 256;  // of a block of the append kernel

// One pool: codes [pages, heads, page, D/2], scale and zero
// [pages, heads, page, D/G].
struct PagedPool {
    uint8_t *c;
    uint16_t *s, *z;
};

struct PagedMap {
    const int32_t *table;  // [B, max_pages]
    const int32_t *len;    // [B]
    const int32_t *cu;     // [B + 1]
    int T, B;
    int max_pages, n_pages, page;
    paged::Divisor div;    // by page
};

struct RopeArgs {
    const int32_t *pos;     // [axes, pos_stride], or null: the cache position
    int64_t pos_stride;
    const float *inv_freq;  // [half], or null: no rotary
    int half;               // pairs of a head row
    int interleaved;        // pairs (2f, 2f + 1) instead of (f, f + half)
    uint32_t axis[8];       // axis of pair f: bits 2 (f % 16) .. + 1 of word f / 16
};

struct AppendArgs {
    const uint16_t *q, *k, *v;  // rows of T tokens; k, v null for the rotary alone
    int64_t q_stride, k_stride, v_stride;  // elements between tokens
    uint16_t *qo;
    int64_t qo_stride;
    PagedPool kp, vp;
    PagedMap map;
    RopeArgs rope;
    int hq, hkv;
    int D, G;
    int rot_k, rot_v;  // Hadamard of the queries and keys, of the values
    float c;           // RN32(1 / sqrt(D))
    float clip;
};

struct PagedAttnArgs {
    const uint16_t *q;
    int64_t q_stride;
    uint16_t *out;
    int64_t out_stride;
    PagedPool kp, vp;
    PagedMap map;
    int hq, hkv, rep;
    int D, G;
    int window, sinks;  // window 0: none
    float sm_scale;
    paged::Which which;  // of paged::Part
    int splits, least;
    float *part_o;       // [rows, hkv, splits, D], rows from paged::part_row on
    float *part_ml;      // [rows, hkv, splits, 2]: maximum (in log2 units), sum
};

// What the scored form has beside: each may be absent.
struct ScoredAttnArgs : PagedAttnArgs {
    float cap;             // of the scores; 0: none
    const float *slopes;   // [hq]: what a score loses for each position of distance
    const int32_t *begin;  // [T]: first token that a row sees (sinks apart)
    const int32_t *end;    // [T]: behind the last one
};

// Row (head 0) of position t of sequence b in the pools, or -1: no page.  Without
// a branch, so that it can be scheduled among other work.
__device__ __forceinline__ int64_t pool_row(const PagedMap &m, int hkv, int b, int t)
{
    const int pi = (int)(__umulhi((uint32_t)t, m.div.mul) >> m.div.sh);
    const bool in = t >= 0 && pi < m.max_pages;
    const int page = m.table[(int64_t)b * m.max_pages + (in ? pi : 0)];
    const int64_t row = (int64_t)page * ((int64_t)hkv * m.page) + (t - pi * m.page);
    return in && (uint32_t)page < (uint32_t)m.n_pages ? row : -1;
}

// The 64 sequences or fewer, from lo on, that the last one of which before(b, cu[b])
// holds is among (it holds up to some b): a 64-way search of cu, one load's latency
// for each power of 64.  Each wave does it for itself.
template <class Before>
__device__ __forceinline__ void search(const PagedMap &m, int &lo, int &n, Before before)
{
    const int lane = threadIdx.x & 63;
    lo = 0;
    n = m.B;
    while (n > 64) {
        const int step = (n + 63) / 64, b = lo + min(lane * step, n - 1);
        const uint64_t held = __ballot(lane * step < n && before(b, m.cu[b]));
        const int i = held ? 63 - __builtin_clzll(held) : 0;
        lo += i * step;
        n = min(step, n - i * step);
    }
}

hipError_t launch_append(const AppendArgs &a, hipStream_t s);
hipError_t launch_paged_attention(const PagedAttnArgs &a, int rows, hipStream_t s);
hipError_t launch_scored_attention(const ScoredAttnArgs &a, int rows, hipStream_t s);
hipError_t launch_large_cap_attention(const ScoredAttnArgs &a, int rows, hipStream_t s);

}  // namespace quarot
