// The pages of the 4-bit KV cache, for gfx950: sequences forked, grown and shrunk, the
// pool compacted, and pages copied.
//
// All of it is integers, and every result is a function of the arguments alone: pages are
// dealt from the lowest free number on, to sequences in order, and sums of references are
// the same in any order.  Tables, lengths and references live on the device and are
// changed in place, so that a captured step goes on from its own results.  Whatever they
// hold, no access leaves its buffer: an entry outside 0 .. n - 1 is no page.
//
// But for the copies, what bounds these calls is latency: a launch, and a chain of
// dependent loads (length, entry, reference) of some 500 ns each.
#include <algorithm>

#include "block_scan.hpp"
#include "pages.hpp"

namespace quarot {
namespace {

constexpr int NT = 1024;  // of the kernels that are one block
constexpr int WAVES = NT / 64;

__device__ __forceinline__ bool is_page(int e, int n)
{
    return (uint32_t)e < (uint32_t)n;
}

// Loads and stores past the CU's own cache, where atomics of this kernel may have been.
__device__ __forceinline__ int fresh(const int32_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void put(int32_t *p, int v)
{
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- fork -------------------------------------------------------------------
//
// A block takes C columns of the table: all rows of them in LDS, then each row as its
// parent's was.  No other block looks at its columns, so that rows can change places in
// place; the first block moves the lengths as well.  An entry that stays costs a load and
// nothing else.  Columns of 16 bytes a row keep enough blocks for a table of some hundred
// columns; wider strips only where there are 64 blocks of them all the same.
template <int C>
__global__ __launch_bounds__(256) void k_pages_fork(ForkArgs a)
{
    extern __shared__ int strip[];  // [B][C]
    const int j0 = blockIdx.x * C, cols = min(C, a.P - j0);
    for (int i = threadIdx.x; i < a.B * C; i += 256) {
        const int c = i % C;
        strip[i] = c < cols ? a.table[(int64_t)(i / C) * a.P + j0 + c] : -1;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.B * C; i += 256) {
        const int b = i / C, c = i % C, p = a.parent[b];
        const int was = strip[i], now = is_page(p, a.B) ? strip[p * C + c] : -1;
        if (was == now || c >= cols)
            continue;
        a.table[(int64_t)b * a.P + j0 + c] = now;
        if (is_page(was, a.n))
            atomicSub(a.refs + was, 1);
        if (is_page(now, a.n))
            atomicAdd(a.refs + now, 1);
    }
    if (blockIdx.x == 0) {
        __syncthreads();
        for (int b = threadIdx.x; b < a.B; b += 256)
            strip[b] = a.lens[b];
        __syncthreads();
        for (int b = threadIdx.x; b < a.B; b += 256) {
            const int p = a.parent[b];
            a.lens[b] = is_page(p, a.B) ? strip[p] : 0;
        }
    }
}

// ---- what the kernels of one block share ------------------------------------

// Pages base .. base + NT * PAGES_EACH - 1 of a pool, PAGES_EACH * 64 in a row to each
// wave: bit k of `yes` of a lane is page first + 64 k + lane.  All loads are on their way
// at once.
constexpr int PAGES_EACH = 16;

struct Tile {
    int64_t first;  // page of this lane
    int r[PAGES_EACH];

    __device__ __forceinline__ Tile(const int32_t *refs, int64_t base, int n)
    {
        first = base + (int64_t)(threadIdx.x >> 6) * 64 * PAGES_EACH + (threadIdx.x & 63);
#pragma unroll
        for (int k = 0; k < PAGES_EACH; ++k)
            r[k] = first + 64 * k < n ? refs[first + 64 * k] : 0;
    }
    template <class Test>
    __device__ __forceinline__ int count(int n, uint32_t &yes, Test test) const
    {
        yes = 0;
        int count = 0;
#pragma unroll
        for (int k = 0; k < PAGES_EACH; ++k) {
            const bool t = first + 64 * k < n && test((int)(first + 64 * k), r[k]);
            yes |= t ? 1u << k : 0u;
            count += __builtin_popcountll(__ballot(t));
        }
        return count;
    }
    // Calls f(page, rank) for each page of `yes`, the wave's first at rank.
    template <class F>
    __device__ __forceinline__ void each(uint32_t yes, int rank, F f) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll 1
        for (int k = 0; k < PAGES_EACH; ++k) {  // (its instructions are fetched once)
            const bool t = yes >> k & 1;
            const uint64_t m = __ballot(t);
            if (t)
                f((int)(first + 64 * k), rank + __builtin_popcountll(m & ((1ull << lane) - 1)));
            rank += __builtin_popcountll(m);
        }
    }
};

// ---- reserve ----------------------------------------------------------------
//
// One block.  What a sequence grows by: entries from .. to - 1 hold nothing but new
// tokens, entry `old` (or -1) older ones before them.
struct Growth {
    int len, n;
    int64_t after;
    int old, from, to;
};

__device__ __forceinline__ Growth growth(const ReserveArgs &a, int b)
{
    Growth g = {};
    g.old = -1;
    if (b >= a.B)
        return g;
    g.len = max(0, a.lens[b]);
    g.n = a.n_new[b];
    g.after = max((int64_t)0, (int64_t)g.len + g.n);
    const int whole = (int)(__umulhi((uint32_t)g.len, a.div.mul) >> a.div.sh);
    const bool part = g.len - whole * a.page != 0;
    const int64_t cap = (int64_t)a.P * a.page;
    const int after = (int)min(g.after, cap);
    const int to = (int)(__umulhi((uint32_t)(after + a.page - 1), a.div.mul) >> a.div.sh);
    if (g.n > 0) {
        g.old = part && whole < a.P ? whole : -1;
        g.from = whole + part;
        g.to = to;
    } else {  // entries that hold nothing any more
        g.from = to;
        g.to = min(a.P, whole + (int)part);
    }
    return g;
}

// Gives back the entries that the wave's sequences shrink out of, 64 of one at a time.
__device__ __forceinline__ void shrink(const ReserveArgs &a, int b, const Growth &g)
{
    const int lane = threadIdx.x & 63;
    for (uint64_t some = __ballot(g.n < 0 && g.from < g.to); some; some &= some - 1) {
        const int i = __builtin_ctzll(some), to = __builtin_amdgcn_readlane(g.to, i);
        int32_t *row = a.table + (int64_t)__builtin_amdgcn_readlane(b, i) * a.P;
        for (int j = __builtin_amdgcn_readlane(g.from, i) + lane; j < to; j += 64) {
            const int e = row[j];
            row[j] = -1;
            if (is_page(e, a.n))
                atomicSub(a.refs + e, 1);
        }
    }
}

// What missing[0] says of pages that are lacking.
__device__ __forceinline__ int lacking(int64_t pages)
{
    return (int)min(max(pages, (int64_t)0), (int64_t)0x7FFFFFFF);
}

// Entry `old` of sequence b as it stands, where it is a page that others hold as well.
__device__ __forceinline__ int shared_page(const ReserveArgs &a, int b, const Growth &g)
{
    if (g.old < 0)
        return -1;
    const int e = a.table[(int64_t)b * a.P + g.old];
    return is_page(e, a.n) && a.refs[e] > 1 ? e : -1;
}

__global__ __launch_bounds__(NT) void k_pages_reserve(ReserveArgs a)
{
    __shared__ int at[PAGES_MAX_BATCH];  // fresh pages of the sequences before each
    __shared__ int sums[WAVES];
    __shared__ int64_t sums8[WAVES];
    const int tid = threadIdx.x, lane = tid & 63;
    int32_t *count = a.ws, *lowest = a.ws + a.n, *list = a.ws + 2 * (int64_t)a.n, *left = a.ws + 3 * (int64_t)a.n;

    // A shared page that all its sequences are about to write on stays with the lowest of
    // them: counted by page, in cells that are cleared first.
    bool any = false;
    for (int b = tid; b < a.B; b += NT) {
        const int e = shared_page(a, b, growth(a, b));
        if (e >= 0) {
            put(count + e, 0);
            put(lowest + e, a.B);
            any = true;
        }
    }
    if (__syncthreads_or(any)) {
        __threadfence();
        for (int b = tid; b < a.B; b += NT) {
            const int e = shared_page(a, b, growth(a, b));
            if (e >= 0) {
                atomicAdd(count + e, 1);
                atomicMin(lowest + e, b);
            }
        }
        __threadfence();
        __syncthreads();
    }
    auto copied = [&](int b, const Growth &g) {  // the page that b has to copy, or -1
        const int e = shared_page(a, b, g);
        return e >= 0 && fresh(count + e) == a.refs[e] && fresh(lowest + e) == b ? -1 : e;
    };
    // Calls f(j, needed, rank) for the entries from .. to - 1 of each growing sequence of
    // the wave's, 64 at a time; the sequence's lane gets how many were needed.
    auto entries = [&](int b, const Growth &g, int rank0, auto f) {
        int mine = 0;
        for (uint64_t left_ = __ballot(g.n > 0 && g.from < g.to); left_; left_ &= left_ - 1) {
            const int i = __builtin_ctzll(left_);
            const int from = __builtin_amdgcn_readlane(g.from, i), to = __builtin_amdgcn_readlane(g.to, i);
            const int bb = __builtin_amdgcn_readlane(b, i);
            int rank = __builtin_amdgcn_readlane(rank0, i);
            const int first = rank;
            for (int j0 = from; j0 < to; j0 += 64) {
                const int j = j0 + lane;
                const int e = j < to ? a.table[(int64_t)bb * a.P + j] : -1;
                const bool page = is_page(e, a.n);
                const bool need = j < to && !(page && a.refs[page ? e : 0] <= 1);
                const uint64_t m = __ballot(need);
                if (need)
                    f((int64_t)bb * a.P + j, page ? e : -1, rank + __builtin_popcountll(m & ((1ull << lane) - 1)));
                rank += __builtin_popcountll(m);
            }
            mine += lane == i ? rank - first : 0;
        }
        return mine;
    };

    int64_t total = 0, rows = 0;
    bool past = false;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int b = b0 + tid;
        const Growth g = growth(a, b);
        int need = copied(b, g) >= 0;
        need += entries(b, g, 0, [](int64_t, int, int) {});
        int64_t all;
        const int64_t before = total + block_scan<WAVES>((int64_t)need, sums8, all);
        if (b < a.B)
            at[b] = (int)before;
        total += all;
        past |= g.after > (int64_t)a.P * a.page;
        rows += max(0, g.n);
    }
    // (new tokens of all sequences, as a batch has them at most)
    int64_t tokens;
    block_scan<WAVES>(rows, sums8, tokens);
    past = __syncthreads_or(past) || tokens > 1 << 30;

    int found = 0;
    for (int64_t base = 0; base < a.n && found < total; base += NT * PAGES_EACH) {
        const Tile tile(a.refs, base, a.n);
        uint32_t yes;
        const int mine = tile.count(a.n, yes, [](int, int r) { return r == 0; });
        int all;
        // (a wave's count is the same in its lanes: its first lane brings it)
        const int before = block_scan<WAVES>(lane == 0 ? mine : 0, sums, all);
        tile.each(yes, found + __builtin_amdgcn_readfirstlane(before), [&](int page, int rank) {
            if (rank < total)
                list[rank] = page;
        });
        found += all;
    }
    __syncthreads();
    const bool done = !past && found >= total;

    // the table and the copies; references change when all of them have been read
    int cu = 0;
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int b = b0 + tid;
        const Growth g = growth(a, b);
        int all;
        const int before = cu + block_scan<WAVES>(done ? max(0, g.n) : 0, sums, all);
        cu += all;
        int src = -1, dst = -1, rank = 0;
        if (b < a.B && done) {
            rank = at[b];
            src = copied(b, g);
            if (src >= 0) {
                dst = list[rank];
                left[rank++] = src;
                a.table[(int64_t)b * a.P + g.old] = dst;
            }
        }
        if (done)
            entries(b, g, rank, [&](int64_t i, int was, int r) {
                a.table[i] = list[r];
                left[r] = was;
            });
        if (b < a.B) {
            a.cu[b] = before;
            a.src[b] = src;
            a.dst[b] = dst;
        }
    }
    if (tid == 0) {
        a.cu[a.B] = cu;
        *a.missing = past ? -1 : lacking(total - found);
    }
    if (!done)
        return;
    __syncthreads();
    for (int i = tid; i < total; i += NT) {
        const int was = left[i];
        put(a.refs + list[i], 1);
        if (was >= 0)
            atomicSub(a.refs + was, 1);
    }
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int b = b0 + tid;
        const Growth g = growth(a, b);
        shrink(a, b, g);
        if (b < a.B)
            a.lens[b] = (int)g.after;
    }
}

// The same for batches of a sequence a thread: what was read stays in registers, sharers
// find each other in a table in LDS, and the first free pages are read while the sequences
// are.  (64 sequences that grow by a token: 12.4 us by the kernel above; 256 beams, most on
// a shared page, 21.7.)
constexpr int SLOTS = 2 * NT;  // of that table
constexpr int FREE = 2048;     // pages of the list that are kept in LDS

__global__ __launch_bounds__(NT) void k_pages_reserve_few(ReserveArgs a)
{
    __shared__ int slot_page[SLOTS], slot_count[SLOTS], slot_lowest[SLOTS];
    __shared__ int64_t sums[WAVES];
    __shared__ int sums1[WAVES], near[FREE];
    const int b = threadIdx.x, lane = b & 63;
    int32_t *list = a.ws + 2 * (int64_t)a.n, *left = a.ws + 3 * (int64_t)a.n;
    const Tile head(a.refs, 0, a.n);
    const Growth g = growth(a, b);
    // the entry with older tokens, and the first with new ones alone
    const int64_t row = (int64_t)b * a.P;
    const bool grows = g.n > 0 && g.from < g.to;
    const int e0 = g.old >= 0 ? a.table[row + g.old] : -1;
    const int e1 = grows ? a.table[row + g.from] : -1;
    const int r0 = is_page(e0, a.n) ? a.refs[e0] : 0, r1 = is_page(e1, a.n) ? a.refs[e1] : 0;
    for (int i = b; i < SLOTS; i += NT) {
        slot_page[i] = -1;
        slot_count[i] = 0;
        slot_lowest[i] = NT;
    }
    __syncthreads();
    int slot = -1;
    if (r0 > 1) {  // (a slot is free: there are twice as many as sequences)
        slot = (uint32_t)e0 * 2654435769u >> 21;
        static_assert(SLOTS == 1 << 11, "the hash's bits");
        for (int held; (held = atomicCAS(&slot_page[slot], -1, e0)) != -1 && held != e0;)
            slot = (slot + 1) % SLOTS;
        atomicAdd(&slot_count[slot], 1);
        atomicMin(&slot_lowest[slot], b);
    }
    __syncthreads();
    const bool copies = slot >= 0 && !(slot_count[slot] == r0 && slot_lowest[slot] == b);
    const bool fresh1 = grows && !(is_page(e1, a.n) && r1 <= 1);
    // Calls f(index, page or -1, rank) for the needed entries behind the first of each
    // sequence of the wave's, 64 at a time; the sequence's lane gets how many they were.
    auto rest = [&](int rank0, auto f) {
        int mine = 0;
        for (uint64_t some = __ballot(grows && g.from + 1 < g.to); some; some &= some - 1) {
            const int i = __builtin_ctzll(some);
            const int from = __builtin_amdgcn_readlane(g.from, i) + 1, to = __builtin_amdgcn_readlane(g.to, i);
            const int64_t base = (int64_t)__builtin_amdgcn_readlane(b, i) * a.P;
            const int first = __builtin_amdgcn_readlane(rank0, i);
            int rank = first;
            for (int j0 = from; j0 < to; j0 += 64) {
                const int j = j0 + lane;
                const int e = j < to ? a.table[base + j] : -1;
                const bool page = is_page(e, a.n);
                const bool need = j < to && !(page && a.refs[page ? e : 0] <= 1);
                const uint64_t m = __ballot(need);
                if (need)
                    f(base + j, page ? e : -1, rank + __builtin_popcountll(m & ((1ull << lane) - 1)));
                rank += __builtin_popcountll(m);
            }
            mine += lane == i ? rank - first : 0;
        }
        return mine;
    };
    const int need = copies + fresh1 + rest(0, [](int64_t, int, int) {});
    int64_t total, tokens;
    const int mine = (int)block_scan<WAVES>((int64_t)need, sums, total);
    const int cu = (int)block_scan<WAVES>((int64_t)max(0, g.n), sums, tokens);
    const bool past = __syncthreads_or(g.after > (int64_t)a.P * a.page) || tokens > 1 << 30;

    int found = 0;
    for (int64_t base = 0; base < a.n && found < total; base += NT * PAGES_EACH) {
        const Tile tile = base ? Tile(a.refs, base, a.n) : head;
        uint32_t yes;
        const int count = tile.count(a.n, yes, [](int, int r) { return r == 0; });
        int some;
        const int first = found + __builtin_amdgcn_readfirstlane(block_scan<WAVES>(lane == 0 ? count : 0, sums1, some));
        if (first < total)
            tile.each(yes, first, [&](int page, int rank) {
                if (rank < FREE)
                    near[rank] = page;
                else if (rank < total)
                    list[rank] = page;
            });
        found += some;
    }
    const bool done = !past && found >= total;
    __syncthreads();
    auto page_of = [&](int rank) { return rank < FREE ? near[rank] : list[rank]; };
    int rank = mine, dst = -1, page1 = -1;
    if (done) {
        if (copies) {
            dst = page_of(rank++);
            a.table[row + g.old] = dst;
        }
        if (fresh1) {
            page1 = page_of(rank++);
            a.table[row + g.from] = page1;
        }
        rest(rank, [&](int64_t i, int was, int r) {
            a.table[i] = page_of(r);
            left[r] = was;
        });
    }
    if (b < a.B) {
        a.cu[b] = done ? cu : 0;
        a.src[b] = dst >= 0 ? e0 : -1;
        a.dst[b] = dst;
    }
    if (b == 0) {
        a.cu[a.B] = done ? (int)tokens : 0;
        *a.missing = past ? -1 : lacking(total - found);
    }
    if (!done)
        return;
    __syncthreads();  // references change once all have been read
    if (dst >= 0) {
        put(a.refs + dst, 1);
        atomicSub(a.refs + e0, 1);
    }
    if (page1 >= 0) {
        put(a.refs + page1, 1);
        if (is_page(e1, a.n))
            atomicSub(a.refs + e1, 1);
    }
    // the others, by their ranks: those behind each sequence's own two
    const int own = copies + fresh1;
    for (uint64_t some = __ballot(need > own); some; some &= some - 1) {
        const int i = __builtin_ctzll(some);
        const int first = __builtin_amdgcn_readlane(mine + own, i), end = __builtin_amdgcn_readlane(mine + need, i);
        for (int r = first + lane; r < end; r += 64) {
            put(a.refs + page_of(r), 1);
            const int was = left[r];
            if (was >= 0)
                atomicSub(a.refs + was, 1);
        }
    }
    shrink(a, b, g);
    if (b < a.B)
        a.lens[b] = (int)g.after;
}

// ---- compact ----------------------------------------------------------------
//
// With L live pages, those numbered L and more move to the free numbers below L, in order;
// no page is both, so that all of them can be copied at once.  One block finds them; then
// the table's entries follow.
__global__ __launch_bounds__(NT) void k_pages_compact(CompactArgs a)
{
    __shared__ int sums[WAVES];
    __shared__ int64_t sums2[WAVES];
    const int tid = threadIdx.x, lane = tid & 63;
    const Tile head(a.refs, 0, a.n);
    int live = 0;
    for (int64_t base = 0; base < a.n; base += NT * PAGES_EACH) {
        const Tile tile = base ? Tile(a.refs, base, a.n) : head;
        uint32_t yes;
        const int mine = tile.count(a.n, yes, [](int, int r) { return r > 0; });
        int all;
        block_scan<WAVES>(lane == 0 ? mine : 0, sums, all);
        live += all;
    }
    int64_t pairs = 0;  // sources below, destinations from bit 32 on
    for (int64_t base = 0; base < a.n; base += NT * PAGES_EACH) {
        const Tile tile = base ? Tile(a.refs, base, a.n) : head;
        uint32_t from, to;
        const int64_t ms = tile.count(a.n, from, [&](int i, int r) { return r > 0 && i >= live; });
        const int64_t md = tile.count(a.n, to, [&](int i, int r) { return r <= 0 && i < live; });
        int64_t all;
        const int64_t before = pairs + block_scan<WAVES>(lane == 0 ? ms | md << 32 : 0, sums2, all);
        const int bs = __builtin_amdgcn_readfirstlane((int)before), bd = __builtin_amdgcn_readfirstlane((int)(before >> 32));
        tile.each(from, bs, [&](int p, int r) { a.src[r] = p; });
        tile.each(to, bd, [&](int p, int r) { a.dst[r] = p; });
        pairs += all;
    }
    const int moves = (int)pairs;
    for (int64_t i = live + tid; i < a.n; i += NT)
        a.ws[i] = (int)i;
    for (int i = moves + tid; i < a.n / 2; i += NT)
        a.src[i] = a.dst[i] = -1;
    if (tid == 0)
        *a.live = live;
    __syncthreads();
    for (int i = tid; i < moves; i += NT) {
        const int s = a.src[i], d = a.dst[i];
        a.ws[s] = d;
        a.refs[d] = a.refs[s];
        a.refs[s] = 0;
    }
}

__global__ __launch_bounds__(256) void k_pages_follow(CompactArgs a)
{
    const int live = *a.live;
    const int64_t of = (int64_t)a.B * a.P;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < of; i += (int64_t)gridDim.x * 256) {
        const int e = a.table[i];
        if (e >= live && e < a.n)
            a.table[i] = a.ws[e];
    }
}

// ---- copy -------------------------------------------------------------------
//
// A block moves 8 KB of a page's codes, or all of its scales and zeros.  Bound by memory.
constexpr int COPY_BYTES = 8192;

__device__ __forceinline__ void move(const uint8_t *base, int64_t from, int64_t to, int64_t bytes)
{
    const uint4 *s = reinterpret_cast<const uint4 *>(base + from);
    uint4 *d = reinterpret_cast<uint4 *>(const_cast<uint8_t *>(base) + to);
    for (int i = threadIdx.x; i < bytes / 16; i += 256)
        d[i] = s[i];
}

__global__ __launch_bounds__(256) void k_pages_copy(CopyArgs a, int pieces)
{
    const int per = (pieces - 1) / 2;
    for (int64_t x = blockIdx.x; x < (int64_t)a.count * pieces; x += gridDim.x) {
        const int i = (int)(x / pieces), piece = (int)(x % pieces);
        const int src = a.src[i], dst = a.dst[i];
        if (!is_page(src, a.n) || !is_page(dst, a.n) || src == dst)
            continue;
        const int64_t cs = src * a.const_bytes, cd = dst * a.const_bytes;
        if (piece == pieces - 1) {
            move(reinterpret_cast<const uint8_t *>(a.kp.s), cs, cd, a.const_bytes);
            move(reinterpret_cast<const uint8_t *>(a.kp.z), cs, cd, a.const_bytes);
            move(reinterpret_cast<const uint8_t *>(a.vp.s), cs, cd, a.const_bytes);
            move(reinterpret_cast<const uint8_t *>(a.vp.z), cs, cd, a.const_bytes);
        } else {
            const int64_t off = (int64_t)(piece % per) * COPY_BYTES;
            move(piece < per ? a.kp.c : a.vp.c, src * a.code_bytes + off, dst * a.code_bytes + off,
                 min((int64_t)COPY_BYTES, a.code_bytes - off));
        }
    }
}

}  // namespace

hipError_t launch_pages_fork(const ForkArgs &a, hipStream_t s)
{
    // 64 KB of LDS at most
    const int fit = 16384 / a.B;
    auto go = [&](auto C) {
        constexpr int c = decltype(C)::value;
        hipLaunchKernelGGL(k_pages_fork<c>, dim3((unsigned)((a.P + c - 1) / c)), dim3(256),
                           (size_t)a.B * c * sizeof(int), s, a);
        return hipGetLastError();
    };
    if (fit >= 16 && a.P >= 64 * 16)
        return go(std::integral_constant<int, 16>());
    if (fit >= 4)
        return go(std::integral_constant<int, 4>());
    return go(std::integral_constant<int, 1>());
}

hipError_t launch_pages_reserve(const ReserveArgs &a, hipStream_t s)
{
    if (a.B <= NT)
        hipLaunchKernelGGL(k_pages_reserve_few, dim3(1), dim3(NT), 0, s, a);
    else
        hipLaunchKernelGGL(k_pages_reserve, dim3(1), dim3(NT), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL(k_pages_compact, dim3(1), dim3(NT), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const int64_t blocks = std::min<int64_t>(((int64_t)a.B * a.P + 255) / 256, 1024);
    hipLaunchKernelGGL(k_pages_follow, dim3((unsigned)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyArgs &a, hipStream_t s)
{
    const int64_t per = (a.code_bytes + COPY_BYTES - 1) / COPY_BYTES, pieces = 2 * per + 1;
    const int64_t blocks = std::min<int64_t>(a.count * pieces, 1 << 20);
    hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)blocks), dim3(256), 0, s, a, (int)pieces);
    return hipGetLastError();
}

}  // namespace quarot
