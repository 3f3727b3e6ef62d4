// Sampling of the next token of each row of logits, for gfx950.
//
// With m the largest logit and T the temperature a token's weight is w = exp((l - m) / T).
// Tokens in the order of their logits (the lower index first where they are equal) are
// cut three times: to the first k, to the shortest beginning whose weights sum up to p of
// what the first cut left, and to weights of min_p and more.  The token is the first one
// in the order of the vocabulary at which the sum of the weights that are left passes u of
// their total.
//
// Weights are whole numbers, rint(w 2^log2_one) from a binary64 exponential (relative
// error below 2e-13), and all sums are sums of those: exact, whatever their order, and so
// is every decision.  2^log2_one lets the sum of a vocabulary stay below 2^63 (a
// vocabulary of 2^17: 2^45), so that a weight that becomes 0 is below 2^-46 of the
// largest.
//
// A block of 16 waves takes a row.  What a cut leaves is mostly few tokens: a list of up to
// LIST of them in LDS, in which the cuts, and the draw, are searches of some tokens a
// thread.
//   k      The largest logits of groups of eight, counted by steps of (m - l) / T, give a
//          logit that k groups reach, and so at least k tokens and hardly more.
//   p      A histogram of the weights of all tokens by their exponents, in 1/32 of a factor
//          of 2, gives a logit that the cut does not pass, and how many tokens lie above it.
//   min_p  is a least logit.
// A search sums amounts (ones or weights) in 2048 bins, over the keys of the logits, and
// divides the bin that holds the target again; few tokens are ranked against each other,
// equal ones by their numbers.  Rows with more left than a list holds are searched in the
// same way as a whole, and drawn from by the sums of what is left, by sixteenths of the row
// and then by tiles of the one that the draw falls in.
//
// What bounds it: instructions, of 131072 tokens a microsecond for each one a token of the
// row's CU.  A pass for the largest logit or for a list is a handful (two fp16 at once, or
// groups that hold none left out), weighing a token 32 to 40, 13 of them in binary64.  All of it is
// inlined: where a function took the row or the cut by reference they lived in scratch memory,
// and the loops waited for all their loads at each use (a share of 0.98 of 50003 tokens, 61 us
// before and 42 without; conditions as masks of a wave, no branches or selects, 39).
#include <algorithm>

#include "block_scan.hpp"
#include "sample.hpp"

namespace quarot {
namespace {

constexpr int NT = 1024, WAVES = NT / 64;
constexpr int BINS = 2048;
constexpr int TILE = 512;  // elements of a wave's step: 8 a lane
constexpr int TILES = SAMPLE_MAX_VOCAB / TILE + 1;
constexpr int LIST = 8192;    // tokens in LDS
constexpr int SOME = 512;     // of them to be ranked
constexpr int STEPS = 256;    // of a factor of 2 in the table of powers

typedef unsigned long long u64;

template <int N>
struct Tokens {
    u64 w[N];
    float l[N];
    int at[N];
};

struct Shared {
    union {
        u64 bins[BINS];   // a histogram
        u64 tile[TILES];  // or sums of the tiles
    };
    u64 sums[WAVES];
    double pow2[STEPS];
    float edge[2][8];  // the row's first and last eight, where they are not eight
    Tokens<LIST> list;
    union {
        Tokens<SOME> some;
        uint32_t count[BINS];  // tokens of a histogram's bins
    };
    uint32_t kmin, found, bin;
    u64 before;
    int token;
};

constexpr float MOST = 0x1.FFFFFEp127f;

// Whole numbers in the order of the logits, one for each number: with a number for -0 of
// its own, the one before that of 0 would be no smaller logit.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l + 0.0f);  // (no -0)
    return b & 0x80000000u ? 0u - b : b | 0x80000000u;
}

__device__ __forceinline__ float of_key(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : 0u - k);
}

template <class T>
struct Row {
    const T *p;
    int V, head, tiles;  // 16-byte loads begin `head` elements before the row
    const float (*edge)[8];

    __device__ __forceinline__ Row(const SampleArgs &a, int64_t row, Shared &s)
    {
        p = static_cast<const T *>(a.logits) + row * a.stride;
        V = a.V;
        head = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % (16 / sizeof(T)));
        tiles = (V + head + TILE - 1) / TILE;
        edge = s.edge;
        if (threadIdx.x < 16) {  // the eight from -head on, and the last eight
            const int last = threadIdx.x >> 3, i = (last ? (V + head - 1) / 8 * 8 : 0) + (threadIdx.x & 7) - head;
            float l = -__builtin_inff();
            if (i >= 0 && i < V) {
                if constexpr (sizeof(T) == 2)
                    l = h2f(p[i]);
                else
                    l = p[i];
            }
            s.edge[last][threadIdx.x & 7] = l;
        }
        __syncthreads();
    }
    __device__ __forceinline__ int index(int tile, int e) const
    {
        return tile * TILE + (threadIdx.x & 63) * 8 + e - head;
    }
    struct Raw {
        uint4 v[sizeof(T) / 2];
    };
    __device__ __forceinline__ void fetch(int tile, Raw &x) const
    {
        const int i = index(tile, 0);
        if (i >= 0 && i + 8 <= V)
#pragma unroll
            for (size_t k = 0; k < sizeof(T) / 2; ++k)
                x.v[k] = reinterpret_cast<const uint4 *>(p + i)[k];
    }
    // As they come (no comparison holds of what is no number); -inf outside the row.
    __device__ __forceinline__ void values(int tile, const Raw &x, float (&l)[8]) const
    {
        const int i = index(tile, 0);
        if (i >= 0 && i + 8 <= V) {
            uint32_t w[2 * sizeof(T)];
            __builtin_memcpy(w, x.v, sizeof(w));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                l[e] = sizeof(T) == 2 ? h2f((uint16_t)(w[e / 2] >> (16 * (e & 1)))) : __uint_as_float(w[e]);
            return;
        }
        const bool none = i >= V;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            l[e] = none ? -__builtin_inff() : edge[i >= 0][e];
    }
    // The largest logit of a lane's eight.
    __device__ __forceinline__ float top(int tile, const Raw &x) const
    {
        const int i = index(tile, 0);
        if (sizeof(T) == 2 && i >= 0 && i + 8 <= V) {
            typedef _Float16 h2v __attribute__((ext_vector_type(2)));
            h2v h[4];
            __builtin_memcpy(h, x.v, sizeof(h));
            const h2v a = __builtin_elementwise_max(__builtin_elementwise_max(h[0], h[1]),
                                                    __builtin_elementwise_max(h[2], h[3]));
            return fmaxf((float)a[0], (float)a[1]);
        }
        float l[8];
        values(tile, x, l);
        return fmaxf(fmaxf(fmaxf(l[0], l[1]), fmaxf(l[2], l[3])), fmaxf(fmaxf(l[4], l[5]), fmaxf(l[6], l[7])));
    }
    __device__ __forceinline__ void load(int tile, float (&l)[8]) const
    {
        Raw x;
        fetch(tile, x);
        values(tile, x, l);
    }
    // f(tile, raw) of the tiles of this wave, the next AHEAD of which are on their way (a
    // row passes by from its XCD's L2 after the first time).  The body stays one copy: with
    // eight tiles unrolled, a pass that weighs every token waited for its instructions, 115
    // us for 131072 tokens instead of 33.
    static constexpr int AHEAD = 16 / (int)sizeof(T) / 2;
    // of tiles first, first + step, .. before end
    template <class F>
    __device__ __forceinline__ void raws(int first, int end, int step, F f) const
    {
        Raw x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (first + k * step < end)
                fetch(first + k * step, x[k]);
#pragma unroll 1
        for (int t = first; t < end; t += step) {
            const Raw now = x[0];
#pragma unroll
            for (int k = 1; k < AHEAD; ++k)
                x[k - 1] = x[k];
            if (t + AHEAD * step < end)
                fetch(t + AHEAD * step, x[AHEAD - 1]);
            f(t, now);
        }
    }
    template <class F>
    __device__ __forceinline__ void tops(F f) const
    {
        raws(threadIdx.x >> 6, tiles, WAVES, [&](int t, const Raw &x) { f(top(t, x)); });
    }
    // f(tile, logits)
    template <class F>
    __device__ __forceinline__ void each(int first, int end, int step, F f) const
    {
        raws(first, end, step, [&](int t, const Raw &x) {
            float l[8];
            values(t, x, l);
            f(t, l);
        });
    }
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        each(threadIdx.x >> 6, tiles, WAVES, f);
    }
    // of tiles with a logit of `from` and more
    template <class F>
    __device__ __forceinline__ void each_from(float from, F f) const
    {
        raws(threadIdx.x >> 6, tiles, WAVES, [&](int t, const Raw &x) {
            if (!__any(top(t, x) >= from))
                return;
            float l[8];
            values(t, x, l);
            f(t, l);
        });
    }
};

__device__ __forceinline__ float block_max(float v, u64 *sums)
{
    static_for<6>([&](auto J) { v = lane_max<J>(v); });
    float *s = reinterpret_cast<float *>(sums);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s[0];
    for (int w = 1; w < WAVES; ++w)
        v = fmaxf(v, s[w]);
    return v;
}

// The weights of a row.
struct Weights {
    float m;       // the largest logit, or binary32's where that is infinite
    double step;   // STEPS log2(e) / T
    float bin;     // bins a unit of logit
    const double *pow2;  // 2^(i / STEPS + log2_one)

    // exp((l - m) / T) 2^log2_one: 2^(n / STEPS) 2^(r / STEPS), |r| <= 1/2, the second by the
    // terms of its series up to the third (the fourth is below 2e-13).  n from the last bits
    // of a sum with 3 2^51.  2^-64 stands for all that is less, and for no number.
    __device__ __forceinline__ double real(float l, int &n) const
    {
        const double x = fmin(fmax(((double)l - (double)m) * step, -64.0 * STEPS), 0.0);
        const double t = x + 0x1.8p52, r = x - (t - 0x1.8p52);
        n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
        constexpr double c = 0.693147180559945309417 / STEPS;
        const double p =
            __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, c * c * c / 6, c * c / 2), c), 1.0);
        const double y = pow2[n & (STEPS - 1)] * p;
        // (far from the ends of the exponent)
        return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, y) + ((int64_t)(n >> 8) << 52));
    }
    __device__ __forceinline__ double real(float l) const
    {
        int n;
        return real(l, n);
    }
    // to a whole number, by a sum with 2^52
    __device__ __forceinline__ u64 whole(float l, int &n) const
    {
        return __builtin_bit_cast(uint64_t, real(l, n) + 0x1p52) & 0xFFFFFFFFFFFFFull;
    }
    __device__ __forceinline__ u64 operator()(float l) const
    {
        int n;
        return whole(l, n);
    }
    // The logit so many steps of the exponent below the largest, nearly.
    __device__ __forceinline__ double down(double steps) const { return (double)m - steps / step; }
    // Bins of the weights: eight steps of the exponent each.
    __device__ __forceinline__ static int bin_of_step(int n) { return std::min(-n >> 3, BINS - 1); }
    __device__ __forceinline__ int weight_bin(float l) const
    {
        int n;
        real(l, n);
        return bin_of_step(n);
    }
    // Bins of the logits: equal steps down to weights of 0, which are BINS and more.
    __device__ __forceinline__ int bin_of(float l) const
    {
        // (by halves of the logits, whose difference is always a number)
        const float x = l >= m ? 0.0f : __builtin_fmaf(l, -0.5f, 0.5f * m) * (2.0f * bin);
        return x < (float)BINS ? (int)x : BINS;  // (what is no number: BINS)
    }
};

// What is left of a row: logits above `cut`, and at it up to index `at` (-1: none, and
// EXACT is not needed).
struct Cut {
    float cut;
    int at;
    template <bool EXACT = true>
    __device__ __forceinline__ bool keeps(float l, int i) const
    {
        // (no branches)
        return EXACT ? (l > cut) | ((l == cut) & (i <= at)) : l > cut;
    }
    // those lanes of a wave of which it holds, of element i + e
    template <bool EXACT>
    __device__ __forceinline__ uint64_t mask(float l, int i, int e) const
    {
        return EXACT ? __ballot(l > cut) | (__ballot(l == cut) & __ballot(i <= at - e)) : __ballot(l > cut);
    }
};

__device__ __forceinline__ bool of_lane(uint64_t mask) { return __builtin_amdgcn_inverse_ballot_w64(mask); }

// How many lanes of the mask are before this one.
__device__ __forceinline__ int lanes_before(uint64_t mask)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// f(std::bool_constant<EXACT>)
template <class F>
__device__ __forceinline__ void with_cut(const Cut &c, F f)
{
    if (c.at < 0)
        f(std::false_type());
    else
        f(std::true_type());
}

// The first bin at which the sum reaches the target, target_of(sum of all), and the sum
// before it, by all threads; false where it never does.
template <class F>
__device__ __forceinline__ bool find(Shared &s, F target_of)
{
    constexpr int E = BINS / NT;
    u64 mine[E], sum = 0, all;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        mine[e] = s.bins[threadIdx.x * E + e];
        sum += mine[e];
    }
    u64 before = block_scan<WAVES>(sum, s.sums, all);
    const u64 target = target_of(all);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (before < target && target <= before + mine[e]) {
            s.bin = threadIdx.x * E + e;
            s.before = before;
        }
        before += mine[e];
    }
    __syncthreads();
    return target <= all;
}

__device__ __forceinline__ void clear(Shared &s)
{
    __syncthreads();
#pragma unroll
    for (int i = threadIdx.x; i < BINS; i += NT)
        s.bins[i] = 0;
    if (threadIdx.x == 0) {
        s.found = 0;
        s.kmin = 0xFFFFFFFFu;
    }
    __syncthreads();
}

// The least logit of which yes() holds, which it does from some logit on and of m: between
// the keys of -inf and of m, first among the NT around a guess (which holds it but where the
// logit is near 0 and m is not), then a thousandth of what is left at a time.  (Four such
// steps and no guess: 2.7 us.)
template <class Yes>
__device__ __forceinline__ float least_logit(Shared &s, float m, double guess, Yes yes)
{
    uint32_t low = key_of(-__builtin_inff()), high = key_of(m);  // not yet, and already
    const uint32_t near = key_of((float)guess);
    uint32_t first = std::max(near, low + NT / 2 + 1) - NT / 2, step = 1;
#pragma unroll 1
    while (high - low > 1) {
        __syncthreads();
        if (threadIdx.x == 0)
            s.kmin = high;
        __syncthreads();
        const uint64_t k = (uint64_t)first + (uint64_t)step * threadIdx.x;
        const uint64_t some = __ballot(k < high && yes(of_key((uint32_t)k)));
        if (some && (threadIdx.x & 63) == (uint32_t)__builtin_ctzll(some))
            atomicMin(&s.kmin, (uint32_t)k);
        __syncthreads();
        // the last of which it did not hold, if it was one of these
        const uint32_t least = s.kmin;
        if (least > first)
            low = std::max(low, least < high ? least - step : std::min(high - 1, first + step * (NT - 1)));
        high = least;
        step = (high - low + NT - 1) / NT;
        first = low + step;
    }
    __syncthreads();
    return of_key(high);
}

// The index of the c-th (from 1) token of the vocabulary with `keeps` (there are as many).
template <class T, class Keeps>
__device__ __forceinline__ int nth(Shared &s, const Row<T> &row, u64 c, Keeps keeps)
{
    row.each([&](int t, const float (&l)[8]) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            n += __builtin_popcountll(__ballot(keeps(l[e], row.index(t, e))));
        if ((threadIdx.x & 63) == 0)
            s.tile[t] = n;
    });
    __syncthreads();
    u64 before = 0;
    for (int t0 = 0; t0 < row.tiles; t0 += NT) {
        const int t = t0 + threadIdx.x;
        const u64 n = t < row.tiles ? s.tile[t] : 0;
        u64 all;
        const u64 b = before + block_scan<WAVES>(n, s.sums, all);
        if (b < c && c <= b + n) {
            s.bin = t;
            s.before = b;
        }
        before += all;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        float l[8];
        const int t = s.bin;
        row.load(t, l);
        int n = 0, mine;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            n += keeps(l[e], row.index(t, e));
        mine = n;
        n = wave_scan(n);
        int left = (int)(c - s.before) - (n - mine);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (keeps(l[e], row.index(t, e)) && --left == 0)
                s.token = row.index(t, e);
    }
    __syncthreads();
    const int at = s.token;
    __syncthreads();
    return at;
}

// What the shortest beginning of a share p sums up to, at least.
__device__ __forceinline__ u64 share_of(float p, u64 all)
{
    const double t = __builtin_ceil((double)p * (double)all);
    return t < 1.0 ? 1 : std::min((u64)t, all);
}

// What the sum of the drawn token and those before it is above.
__device__ __forceinline__ u64 draw(float u, u64 all)
{
    const double share = u > 0.0f ? std::min((double)u, 1.0) * (double)all : 0.0;
    return std::min((u64)share, all - 1);
}

// The tokens of the list with in(x) and an amount, up to SOME of them, in `some`; how many.
template <class In, class A>
__device__ __forceinline__ uint32_t pick(Shared &s, int n, In in, A amount)
{
    for (int x = threadIdx.x; x < n; x += NT) {
        const u64 a = in(x) ? amount(x) : 0;
        if (a) {
            const uint32_t y = atomicAdd(&s.found, 1u);
            if (y < SOME) {
                s.some.w[y] = a;
                s.some.l[y] = s.list.l[x];
                s.some.at[y] = s.list.at[x];
            }
        }
    }
    __syncthreads();
    return s.found;
}

// The first of n tokens of `some`, in the order of their logits or their numbers, at which
// the sum of their amounts reaches target.
template <bool BY_NUMBER>
__device__ __forceinline__ Cut rank(Shared &s, int n, u64 target)
{
    if ((int)threadIdx.x < n) {
        const float l = s.some.l[threadIdx.x];
        const int at = s.some.at[threadIdx.x];
        const u64 mine = s.some.w[threadIdx.x];
        u64 sum = 0;
        for (int x = 0; x < n; ++x) {
            const bool first = s.some.at[x] < at;
            const float y = s.some.l[x];
            sum += (BY_NUMBER ? first : y > l || (y == l && first)) ? s.some.w[x] : 0;
        }
        if (sum < target && target <= sum + mine) {
            s.kmin = __float_as_uint(l);
            s.token = at;
        }
    }
    __syncthreads();
    return Cut{__uint_as_float(s.kmin), s.token};
}

// The token of the list, in the order of the numbers, at which the sum of the amounts
// reaches target_of(their sum), which it does.
template <class A, class F>
__device__ __forceinline__ Cut by_number(Shared &s, int n, int V, A amount, F target_of)
{
    int shift = 0;
    while (V > BINS << shift)
        ++shift;
    static_assert(SAMPLE_MAX_VOCAB / BINS <= SOME, "the numbers of a bin");
    clear(s);
    for (int x = threadIdx.x; x < n; x += NT) {
        const u64 a = amount(x);
        if (a)
            atomicAdd(&s.bins[s.list.at[x] >> shift], a);
    }
    __syncthreads();
    u64 target = 0;
    find(s, [&](u64 all) { return target = target_of(all); });
    const int b = (int)s.bin;
    const u64 left = target - s.before;
    return rank<true>(s, (int)pick(s, n, [&](int x) { return s.list.at[x] >> shift == b; }, amount), left);
}

// Bits to shift a difference of keys by, so that it is a bin.
__device__ __forceinline__ int key_shift(uint32_t range)
{
    return range ? std::max(0, 32 - __builtin_clz(range) - 11) : 0;
}

// A bin of keys up to high: what it leaves of low .. high.
__device__ __forceinline__ void narrow(uint32_t &low, uint32_t &high, uint32_t bin, int shift)
{
    high -= bin << shift;
    const uint32_t first = high - ((1u << shift) - 1);
    low = first > low && first <= high ? first : low;
}

// The cut of the list, in the order of the logits, at which the sum of the amounts reaches
// target_of(their sum); where it does not, all of it.  Its keys lie in low .. high.
template <class A, class F>
__device__ __forceinline__ Cut by_logit(Shared &s, int n, int V, uint32_t low, uint32_t high, A amount, F target_of)
{
    u64 target = 0;
    for (bool first = true;; first = false) {
        const int shift = key_shift(high - low);
        auto key = [&](int x) { return key_of(s.list.l[x]); };
        auto in = [&](int x) { return key(x) >= low && key(x) <= high; };
        clear(s);
        for (int x = threadIdx.x; x < n; x += NT) {
            const u64 a = in(x) ? amount(x) : 0;
            if (a)
                atomicAdd(&s.bins[(high - key(x)) >> shift], a);
        }
        __syncthreads();
        if (!find(s, [&](u64 all) { return first ? target = target_of(all) : target; }))
            return Cut{-__builtin_inff(), -1};
        target -= s.before;
        narrow(low, high, s.bin, shift);
        const uint32_t found = pick(s, n, in, amount);
        if (found <= 64)
            return rank<false>(s, (int)found, target);
        if (low == high)
            return by_number(s, n, V, [&](int x) { return key(x) == low ? amount(x) : 0; },
                             [&](u64) { return target; });
    }
}

// The row's tokens from logit `from` on, of the lanes of in(l, index, e), in any order, as
// the list; how many there are, or more than LIST of them.
template <class T, class In>
__device__ __forceinline__ uint32_t gather(Shared &s, const Row<T> &row, float from, In in)
{
    __syncthreads();
    if (threadIdx.x == 0)
        s.found = 0;
    __syncthreads();
    bool full = false;  // nothing will read the list
    row.each_from(from, [&](int t, const float (&l)[8]) {
        if (full)
            return;
        uint64_t m[8];
        int n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = __ballot(l[e] >= from) & in(l[e], row.index(t, 0), e);
            n += __builtin_popcountll(m[e]);
        }
        if (n == 0)
            return;
        uint32_t base = 0;
        if ((threadIdx.x & 63) == 0)
            base = atomicAdd(&s.found, (uint32_t)n);
        base = __builtin_amdgcn_readfirstlane((int)base);
        full = base + n > LIST;
        if (full)
            return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (m[e] == 0)
                continue;
            if (of_lane(m[e])) {
                const int x = (int)base + lanes_before(m[e]);
                s.list.l[x] = l[e];
                s.list.at[x] = row.index(t, e);
            }
            base += __builtin_popcountll(m[e]);
        }
    });
    __syncthreads();
    return s.found;
}

// Cuts what is left of a row, by its tokens with keys low .. high, to its beginning (by
// logit) whose amounts (1, or the weights) reach target, which they do.
template <bool WEIGHTS, class T>
__device__ __forceinline__ void by_row(Shared &s, const Row<T> &row, const Weights &w, Cut &c, u64 target, uint32_t low, uint32_t high)
{
    for (;;) {
        const float from = of_key(low), to = of_key(high);
        uint32_t n;
        with_cut(c, [&](auto exact) {
            n = gather(s, row, from, [&](float l, int i, int e) {
                return __ballot(l <= to) & (exact ? c.mask<true>(l, i, e) : ~0ull);
            });
        });
        if (n <= LIST) {
            for (uint32_t x = threadIdx.x; x < n; x += NT)
                s.list.w[x] = WEIGHTS ? w(s.list.l[x]) : 1;
            c = by_logit(s, (int)n, row.V, low, high, [&](int x) { return s.list.w[x]; }, [&](u64) { return target; });
            return;
        }
        if (low == high) {  // equal ones: the first in the order of the vocabulary
            const float l = of_key(low);
            const u64 each = WEIGHTS ? w(l) : 1;
            const u64 k = (target + each - 1) / each;
            const Cut was = c;
            c.at = nth(s, row, k, [&](float x, int i) { return x == l && was.keeps(x, i); });
            c.cut = l;
            return;
        }
        const int shift = key_shift(high - low);
        clear(s);
        row.each_from(from, [&](int t, const float (&l)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((l[e] >= from) & (l[e] <= to) & c.keeps(l[e], row.index(t, e)))
                    atomicAdd(&s.bins[(high - key_of(l[e])) >> shift], WEIGHTS ? w(l[e]) : 1);
        });
        __syncthreads();
        find(s, [&](u64) { return target; });
        target -= s.before;
        narrow(low, high, s.bin, shift);
    }
}

template <class T>
__global__ __launch_bounds__(NT) void k_sample(SampleArgs a)
{
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    const Row<T> row(a, r, s);
    const float inf = __builtin_inff();
    float m = -inf;
    row.tops([&](float l) { m = fmaxf(m, l); });
    m = block_max(m, s.sums);
    if (m == -inf) {  // nothing is left to choose
        if (threadIdx.x == 0)
            a.tokens[r] = -1;
        return;
    }
    // (infinite: as a number that leaves every finite logit its whole weight)
    const double temp = std::min(a.temperature ? (double)a.temperature[r] : 1.0, 0x1p1000);
    if (!(temp > 0.0)) {
        if (threadIdx.x == 0)
            s.token = a.V;
        __syncthreads();
        int first = a.V;
        row.each_from(m, [&](int t, const float (&l)[8]) {
#pragma unroll
            for (int e = 7; e >= 0; --e)
                first = l[e] == m ? std::min(first, row.index(t, e)) : first;
        });
        if (first < a.V)
            atomicMin(&s.token, first);
        __syncthreads();
        if (threadIdx.x == 0)
            a.tokens[r] = s.token;
        return;
    }
    if (threadIdx.x < STEPS) {  // the series of exp, up to 2^-60 of it
        const double x = threadIdx.x * (0.693147180559945309417 / STEPS);
        double p = 1.0;
#pragma unroll
        for (int i = 18; i > 0; --i)
            p = __builtin_fma(p * x, 1.0 / i, 1.0);
        s.pow2[threadIdx.x] = __builtin_ldexp(p, a.log2_one);
    }
    Weights w;
    w.m = std::min(m, MOST);
    w.step = STEPS * 1.44269504088896340736 / temp;
    // (at most what binary32 holds: at temperatures below 2e-37 the bins are wider, and what
    // lies past the last of them still weighs nothing)
    w.bin = (float)std::min(BINS / ((a.log2_one + 1.5) * 0.693147180559945309417) / temp, 0.5 * MOST);
    w.pow2 = s.pow2;
    __syncthreads();

    int k = a.top_k ? a.top_k[r] : 0;
    k = k < a.V ? std::max(k, 0) : 0;
    float p = a.top_p ? a.top_p[r] : 1.0f;
    p = p < 1.0f ? p : 1.0f;
    const float mp = a.min_p ? a.min_p[r] : 0.0f;
    float least = -MOST;
    if (mp > 0.0f) {  // (not a number: none)
        const double from = std::min((double)mp, 1.0) * w.pow2[0];
        least = least_logit(s, m, w.down(-std::log2(std::min(mp, 1.0f)) * STEPS),
                            [&](float l) { return w.real(l) >= from; });
    }
    const float u = a.u[r];
    // What is left: by the cut, and once it is few, the list (n tokens with keys low .. high).
    Cut c = {-inf, -1};
    bool listed = false;
    uint32_t n = 0, low = 0, high = 0;
    auto gathered = [&](float from) {
        with_cut(c, [&](auto exact) {
            n = gather(s, row, from, [&](float l, int i, int e) {
                return exact ? c.mask<true>(l, i, e) : ~0ull;
            });
        });
        low = key_of(from);
        high = key_of(m);
        listed = n <= LIST;
        if (listed)
            for (uint32_t x = threadIdx.x; x < n; x += NT)
                s.list.w[x] = w(s.list.l[x]);
    };
    auto weight = [&](int x) { return c.keeps(s.list.l[x], s.list.at[x]) ? s.list.w[x] : 0; };
    if (k > 0) {
        if (k <= LIST) {
            clear(s);
            row.tops([&](float l) {
                const int b = w.bin_of(l);
                if (b < BINS)
                    atomicAdd(&s.bins[b], 1ull);
            });
            __syncthreads();
            const int b = find(s, [&](u64) { return (u64)k; }) ? (int)s.bin : BINS - 1;
            // (all of bin b, and a little of the next: the bin's own rounding is 2^-12 of one)
            gathered(fmaxf(w.m - ((float)b + 1.01f) / w.bin, -MOST));
        }
        if (listed) {
            if (k < (int)n)
                c = by_logit(s, (int)n, row.V, low, high, [](int) { return (u64)1; }, [&](u64) { return (u64)k; });
        } else {
            clear(s);
            row.each([&](int, const float (&l)[8]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int b = w.bin_of(l[e]);
                    if (b < BINS)
                        atomicAdd(&s.bins[b], 1ull);
                }
            });
            __syncthreads();
            if (find(s, [&](u64) { return (u64)k; })) {
                const int b = (int)s.bin;
                const u64 before = s.before;
                auto top = [&](int b) {
                    return least_logit(s, m, w.m - (double)(b + 1) / w.bin, [&](float l) { return w.bin_of(l) <= b; });
                };
                const float from = top(b), to = b ? top(b - 1) : inf;
                by_row<false>(s, row, w, c, k - before, key_of(from), b ? key_of(to) - 1 : key_of(m));
            }
        }
    }
    if (p < 1.0f && listed) {
        c = by_logit(s, (int)n, row.V, low, high, weight, [&](u64 all) { return share_of(p, all); });
    } else if (p < 1.0f) {
        const int nothing = -(a.log2_one + 2) * STEPS;  // (less weighs nothing)
        static_assert(53 * STEPS / 8 < BINS, "their bins");
        clear(s);
        for (int i = threadIdx.x; i < BINS; i += NT)
            s.count[i] = 0;
        __syncthreads();
        with_cut(c, [&](auto exact) {
            row.each([&](int t, const float (&l)[8]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    int step;
                    const u64 x = w.whole(l[e], step);
                    bool some = step >= nothing;
                    if (exact)
                        some &= c.keeps(l[e], row.index(t, e));
                    if (some) {
                        atomicAdd(&s.bins[-step >> 3], x);
                        atomicAdd(&s.count[-step >> 3], 1u);
                    }
                }
            });
        });
        __syncthreads();
        u64 target = 0;
        find(s, [&](u64 all) { return target = share_of(p, all); });
        const int b = (int)s.bin;
        const u64 before = s.before;
        uint32_t some = 0;  // tokens down to the end of the bin
        for (int i = threadIdx.x; i <= b; i += NT)
            some += s.count[i];
        block_scan<WAVES>(some, reinterpret_cast<uint32_t *>(s.sums), some);
        auto top = [&](int b) {
            return least_logit(s, m, w.down(8 * b + 7.5), [&](float l) { return w.weight_bin(l) <= b; });
        };
        const float from = top(b);
        if (some <= LIST)
            gathered(from);
        if (listed)  // (more would be tokens of weight 0, which are not counted)
            c = by_logit(s, (int)n, row.V, low, high, weight, [&](u64) { return target; });
        else
            by_row<true>(s, row, w, c, target - before, key_of(from), b ? key_of(top(b - 1)) - 1 : key_of(m));
    } else if (!listed && least > -MOST) {
        gathered(least);
    }
    if (listed) {
        c = by_number(s, (int)n, row.V, [&](int x) { return s.list.l[x] < least ? 0 : weight(x); },
                      [&](u64 all) { return draw(u, all) + 1; });
        if (threadIdx.x == 0)
            a.tokens[r] = c.at;
        return;
    }

    // What is left, by sixteenths of the row, a wave each.  Where it is few of a tile's
    // tokens they are gathered in LDS, 64 to be weighed at once.
    if (c.cut < least && least > -MOST)
        c = Cut{of_key(key_of(least) - 1), -1};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = (row.tiles + WAVES - 1) / WAVES;
    __syncthreads();
    float *few = reinterpret_cast<float *>(&s.list) + wave * ((int)sizeof(s.list) / WAVES / 4);
    static_assert(sizeof(s.list) / WAVES / 4 >= TILE + 64, "a tile's tokens and what an earlier one left");
    int held = 0;
    u64 mine = 0;
    with_cut(c, [&](auto exact) {
        row.each(wave * per, std::min(row.tiles, (wave + 1) * per), 1, [&](int t, const float (&l)[8]) {
            uint64_t m[8];
            int n = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m[e] = c.mask<exact>(l[e], row.index(t, 0), e);
                n += __builtin_popcountll(m[e]);
            }
            if (n > TILE / 2) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    mine += of_lane(m[e]) ? w(l[e]) : 0;
                return;
            }
            if (n == 0)
                return;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (of_lane(m[e]))
                    few[held + lanes_before(m[e])] = l[e];
                held += __builtin_popcountll(m[e]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (; held >= 64; held -= 64)
                mine += w(few[held - 64 + lane]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        });
    });
    if (lane < held)
        mine += w(few[lane]);
    mine = wave_scan(mine);
    if (lane == 63)
        s.tile[wave] = mine;
    __syncthreads();
    u64 all = 0, before = 0;
    for (int x = 0; x < WAVES; ++x)
        all += s.tile[x];
    const u64 target = draw(u, all);
    int part = 0;
    for (int x = 0; x < WAVES; ++x) {
        const u64 n = s.tile[x];
        if (before + n > target) {
            part = x;
            break;
        }
        before += n;
    }
    __syncthreads();
    // its tiles, and the tile's tokens
    const int first = part * per, end = std::min(row.tiles, first + per);
    row.each(first + wave, end, WAVES, [&](int t, const float (&l)[8]) {
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum += w(l[e]) & (c.keeps(l[e], row.index(t, e)) ? ~0ull : 0);
        sum = wave_scan(sum);
        if (lane == 63)
            s.tile[t] = sum;
    });
    __syncthreads();
    {
        static_assert(TILES / WAVES < NT, "a thread for each");
        const int t = first + threadIdx.x;
        const u64 n = t < end ? s.tile[t] : 0;
        u64 ignore;
        const u64 b = before + block_scan<WAVES>(n, s.sums, ignore);
        if (b <= target && target < b + n) {
            s.bin = t;
            s.before = b;
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        float l[8];
        const int t = s.bin;
        row.load(t, l);
        u64 x[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = w(l[e]) & (c.keeps(l[e], row.index(t, e)) ? ~0ull : 0);
            sum += x[e];
        }
        u64 at = s.before + wave_scan(sum) - sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (at <= target && target < at + x[e])
                a.tokens[r] = row.index(t, e);
            at += x[e];
        }
    }
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, bool f32, int64_t rows, hipStream_t s)
{
    if (f32)
        hipLaunchKernelGGL(k_sample<float>, dim3((unsigned)rows), dim3(NT), 0, s, a);
    else
        hipLaunchKernelGGL(k_sample<uint16_t>, dim3((unsigned)rows), dim3(NT), 0, s, a);
    return hipGetLastError();
}

}  // namespace quarot
