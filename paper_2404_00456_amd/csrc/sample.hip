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
// error below 1e-13), and all sums are sums of those: exact, whatever their order, and so
// is every decision.  2^log2_one lets the sum of a vocabulary stay below 2^63 (a
// vocabulary of 2^17: 2^45), so that a weight that becomes 0 is below 2^-46 of the
// largest.
//
// A block of 16 waves takes a row.  A cut is a search: a histogram over (m - l) / T in
// equal steps, 2048 of them down to weights of 0, tells in which step it falls; where more
// than LIST tokens share that, further histograms over the bits of their logits; those
// that are left are ranked against each other.  Where all of them are equal, the index
// decides, by counting in the order of the vocabulary.
#include <algorithm>

#include "block_scan.hpp"
#include "sample.hpp"

namespace quarot {
namespace {

constexpr int NT = 1024, WAVES = NT / 64;
constexpr int BINS = 2048;
constexpr int TILE = 512;  // elements of a wave's step: 8 a lane
constexpr int TILES = SAMPLE_MAX_VOCAB / TILE + 1;
constexpr int LIST = 512;

typedef unsigned long long u64;

struct Shared {
    u64 weight[BINS];  // of a histogram
    uint32_t count[BINS];
    u64 tile[TILES];   // sums of the tiles
    u64 sums[WAVES];
    double pow2[64];   // 2^(i / 64)
    u64 list_w[LIST];
    uint32_t list_key[LIST], list_at[LIST];
    uint32_t kmin, kmax, found, bin;
    u64 before;
    int token;
};

// A logit as the comparisons take it: no -0, and what is not a number as -inf.
__device__ __forceinline__ float clean(float l)
{
    return l == l ? l + 0.0f : -__builtin_inff();
}

// Whole numbers in the order of the logits.
__device__ __forceinline__ uint32_t key_of(float l)
{
    const uint32_t b = __float_as_uint(l);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float of_key(uint32_t k)
{
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

template <class T>
struct Row {
    const T *p;
    int V, head, tiles;  // 16-byte loads begin `head` elements before the row

    __device__ Row(const SampleArgs &a, int64_t row)
    {
        p = static_cast<const T *>(a.logits) + row * a.stride;
        V = a.V;
        head = (int)(reinterpret_cast<uintptr_t>(p) / sizeof(T) % (16 / sizeof(T)));
        tiles = (V + head + TILE - 1) / TILE;
    }
    __device__ int index(int tile, int e) const
    {
        return tile * TILE + (threadIdx.x & 63) * 8 + e - head;
    }
    // -inf outside the row
    __device__ void load(int tile, float (&l)[8]) const
    {
        const int i = index(tile, 0);
        if (i >= 0 && i + 8 <= V) {
            if constexpr (sizeof(T) == 2) {
                const uint4 v = *reinterpret_cast<const uint4 *>(p + i);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    l[e] = clean(h2f((uint16_t)(w[e / 2] >> (16 * (e & 1)))));
            } else {
                const float4 a = *reinterpret_cast<const float4 *>(p + i);
                const float4 b = *reinterpret_cast<const float4 *>(p + i + 4);
                const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    l[e] = clean(v[e]);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            l[e] = -__builtin_inff();
            if (i + e >= 0 && i + e < V) {
                if constexpr (sizeof(T) == 2)
                    l[e] = clean(h2f(p[i + e]));
                else
                    l[e] = clean(p[i + e]);
            }
        }
    }
    // f(tile, logits) of the tiles of this wave
    template <class F>
    __device__ void each(F f) const
    {
        for (int t = threadIdx.x >> 6; t < tiles; t += WAVES) {
            float l[8];
            load(t, l);
            f(t, l);
        }
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
    float m;
    double step;   // 64 log2(e) / T
    float bin;     // bins a unit of logit
    int one;
    const double *pow2;

    // exp((l - m) / T): 2^(n / 64) 2^(r / 64), |r| <= 1/2, the second by the terms of its
    // series up to the fourth (the fifth is below 4e-14); 0 below 2^-64
    __device__ __forceinline__ double real(float l) const
    {
        const double x = l == m ? 0.0 : ((double)l - (double)m) * step;
        if (!(x > -64.0 * 64.0))
            return 0.0;
        const double n = __builtin_rint(x), r = x - n;
        constexpr double c = 0.693147180559945309417 / 64.0;
        const double p = __builtin_fma(
            r, __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, c * c * c * c / 24, c * c * c / 6), c * c / 2), c), 1.0);
        const int i = (int)n;
        return __builtin_ldexp(pow2[i & 63] * p, i >> 6);
    }
    __device__ __forceinline__ u64 whole(double w) const
    {
        return (u64)__builtin_rint(__builtin_ldexp(w, one));
    }
    __device__ __forceinline__ u64 operator()(float l) const { return whole(real(l)); }
    // BINS and more: a weight of 0
    __device__ __forceinline__ int bin_of(float l) const
    {
        const float x = l == m ? 0.0f : (m - l) * bin;
        return x < (float)BINS ? (int)x : BINS;
    }
};

// What is left of a row: logits above `cut`, and at it up to index `at`.
struct Cut {
    float cut;
    int at;
    __device__ __forceinline__ bool keeps(float l, int i) const { return l > cut || (l == cut && i <= at); }
};

// The first bin at which the sum of `of` reaches target, and the sum before it, by all
// threads; false where it never does.
template <class T>
__device__ __forceinline__ bool find(Shared &s, const T *of, u64 target)
{
    constexpr int E = BINS / NT;
    u64 mine[E], sum = 0, all;
    for (int e = 0; e < E; ++e) {
        mine[e] = of[threadIdx.x * E + e];
        sum += mine[e];
    }
    u64 before = block_scan<WAVES>(sum, s.sums, all);
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
    for (int i = threadIdx.x; i < BINS; i += NT) {
        s.weight[i] = 0;
        s.count[i] = 0;
    }
    __syncthreads();
}

// The index of the c-th (from 1) token of the vocabulary with `keeps` (there are as many).
template <class T, class Keeps>
__device__ int nth(Shared &s, const Row<T> &row, u64 c, Keeps keeps)
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
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(n, d);
            n += (int)threadIdx.x >= d ? y : 0;
        }
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

// Cuts what is left of a row to its beginning (by logit) whose amounts reach `target`, an
// amount being 1 or the token's weight.  The histogram of s is that of all that is left.
template <bool WEIGHTS, class T>
__device__ void cut_to(Shared &s, const Row<T> &row, const Weights &w, Cut &c, u64 target)
{
    auto bins = [&]() { return WEIGHTS ? find(s, s.weight, target) : find(s, s.count, target); };
    if (!bins())
        return;
    // the keys of that bin
    uint32_t bin = s.bin;
    target -= s.before;
    uint32_t n = s.count[bin];
    if (threadIdx.x == 0) {
        s.kmin = 0xFFFFFFFFu;
        s.kmax = 0;
    }
    __syncthreads();
    row.each([&](int t, const float (&l)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (w.bin_of(l[e]) == (int)bin && c.keeps(l[e], row.index(t, e))) {
                atomicMin(&s.kmin, key_of(l[e]));
                atomicMax(&s.kmax, key_of(l[e]));
            }
    });
    __syncthreads();
    uint32_t kmin = s.kmin, kmax = s.kmax;
    while (n > LIST && kmin < kmax) {
        const int bits = 32 - __builtin_clz(kmax - kmin), shift = std::max(0, bits - 11);
        clear(s);
        row.each([&](int t, const float (&l)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t k = key_of(l[e]);
                if (k >= kmin && k <= kmax && c.keeps(l[e], row.index(t, e))) {
                    atomicAdd(&s.count[(kmax - k) >> shift], 1u);
                    if (WEIGHTS)
                        atomicAdd(&s.weight[(kmax - k) >> shift], w(l[e]));
                }
            }
        });
        __syncthreads();
        bins();
        bin = s.bin;
        target -= s.before;
        n = s.count[bin];
        const uint32_t top = kmax - (bin << shift), low = top - ((1u << shift) - 1);
        kmin = low > kmin && low <= top ? low : kmin;
        kmax = top;
    }
    if (kmin == kmax) {  // equal ones: the first in the order of the vocabulary
        const float l = of_key(kmin);
        const u64 each = WEIGHTS ? w(l) : 1;
        const u64 k = (target + each - 1) / each;
        const Cut was = c;
        c.at = nth(s, row, k, [&](float x, int i) { return x == l && was.keeps(x, i); });
        c.cut = l;
        return;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        s.found = 0;
    __syncthreads();
    row.each([&](int t, const float (&l)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t k = key_of(l[e]);
            if (k >= kmin && k <= kmax && c.keeps(l[e], row.index(t, e))) {
                const uint32_t x = atomicAdd(&s.found, 1u);
                if (x < LIST) {
                    s.list_key[x] = k;
                    s.list_at[x] = row.index(t, e);
                    s.list_w[x] = WEIGHTS ? w(l[e]) : 1;
                }
            }
        }
    });
    __syncthreads();
    if (threadIdx.x < n) {
        const uint32_t k = s.list_key[threadIdx.x], at = s.list_at[threadIdx.x];
        const u64 mine = s.list_w[threadIdx.x];
        u64 before = 0;
        for (uint32_t x = 0; x < n; ++x)
            before += s.list_key[x] > k || (s.list_key[x] == k && s.list_at[x] < at) ? s.list_w[x] : 0;
        if (before < target && target <= before + mine) {
            s.kmin = k;
            s.token = at;
        }
    }
    __syncthreads();
    c.cut = of_key(s.kmin);
    c.at = s.token;
    __syncthreads();
}

template <class T>
__global__ __launch_bounds__(NT) void k_sample(SampleArgs a)
{
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    const Row<T> row(a, r);
    const float inf = __builtin_inff();
    float m = -inf;
    row.each([&](int, const float (&l)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            m = fmaxf(m, l[e]);
    });
    m = block_max(m, s.sums);
    if (m == -inf) {  // nothing is left to choose
        if (threadIdx.x == 0)
            a.tokens[r] = -1;
        return;
    }
    const float temp = a.temperature ? a.temperature[r] : 1.0f;
    if (!(temp > 0.0f)) {
        const int at = nth(s, row, 1, [&](float l, int) { return l == m; });
        if (threadIdx.x == 0)
            a.tokens[r] = at;
        return;
    }
    if (threadIdx.x < 64) {  // the series of exp, up to 2^-60 of it
        const double x = threadIdx.x * (0.693147180559945309417 / 64.0);
        double p = 1.0;
        for (int i = 18; i > 0; --i)
            p = __builtin_fma(p, x / i, 1.0);
        s.pow2[threadIdx.x] = p;
    }
    Weights w;
    w.m = m;
    w.step = 64.0 * 1.44269504088896340736 / (double)temp;
    w.one = a.log2_one;
    w.bin = (float)(BINS / ((a.log2_one + 1.5) * 0.693147180559945309417) / (double)temp);
    w.pow2 = s.pow2;

    Cut c = {-inf, -1};
    const int k = a.top_k ? a.top_k[r] : 0;
    if (k > 0 && k < a.V) {
        clear(s);
        row.each([&](int, const float (&l)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int b = w.bin_of(l[e]);
                if (b < BINS)
                    atomicAdd(&s.count[b], 1u);
            }
        });
        __syncthreads();
        cut_to<false>(s, row, w, c, (u64)k);
    }
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    if (p < 1.0f) {
        clear(s);
        u64 sum = 0, all;
        row.each([&](int t, const float (&l)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int b = w.bin_of(l[e]);
                if (b < BINS && c.keeps(l[e], row.index(t, e))) {
                    const u64 x = w(l[e]);
                    atomicAdd(&s.count[b], 1u);
                    atomicAdd(&s.weight[b], x);
                    sum += x;
                }
            }
        });
        block_scan<WAVES>(sum, s.sums, all);
        const double t = __builtin_ceil((double)p * (double)all);
        cut_to<true>(s, row, w, c, t < 1.0 ? 1 : std::min((u64)t, all));
    }
    const double least = a.min_p ? std::min((double)a.min_p[r], 1.0) : 0.0;  // (NaN: none)
    auto left = [&](float l, int i) -> u64 {
        if (!(l > -inf) || !c.keeps(l, i))
            return 0;
        const double x = w.real(l);
        return x < least ? 0 : w.whole(x);
    };
    __syncthreads();
    row.each([&](int t, const float (&l)[8]) {
        u64 sum = 0;
        bool any = false;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            any |= c.keeps(l[e], row.index(t, e));
        if (__any(any)) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum += left(l[e], row.index(t, e));
            for (int d = 1; d < 64; d <<= 1)
                sum += __shfl_xor(sum, d);
        }
        if ((threadIdx.x & 63) == 0)
            s.tile[t] = sum;
    });
    __syncthreads();
    u64 total = 0;
    for (int t = threadIdx.x; t < row.tiles; t += NT)
        total += s.tile[t];
    u64 all;
    block_scan<WAVES>(total, s.sums, all);
    const float u = a.u[r];
    const double share = u > 0.0f ? std::min((double)u, 1.0) * (double)all : 0.0;
    const u64 target = std::min((u64)share, all - 1);  // the first whose sum is above it
    u64 before = 0;
    for (int t0 = 0; t0 < row.tiles; t0 += NT) {
        const int t = t0 + threadIdx.x;
        const u64 n = t < row.tiles ? s.tile[t] : 0;
        u64 step;
        const u64 b = before + block_scan<WAVES>(n, s.sums, step);
        if (b <= target && target < b + n) {
            s.bin = t;
            s.before = b;
        }
        before += step;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        float l[8];
        const int t = s.bin;
        row.load(t, l);
        u64 x[8], sum = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = left(l[e], row.index(t, e));
            sum += x[e];
        }
        u64 upto = sum;
        for (int d = 1; d < 64; d <<= 1) {
            const u64 y = __shfl_up(upto, d);
            upto += (int)threadIdx.x >= d ? y : 0;
        }
        u64 at = s.before + upto - sum;
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
