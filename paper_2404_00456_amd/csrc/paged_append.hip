// Rotary positions, the head's Hadamard, and the 4-bit codes of new keys and
// values straight into the pages of their cache, for gfx950.
//
// A block takes tokens and a share of their heads; a row of D elements is
// D / 8 lanes of 8 consecutive elements (placed as lane_pos says, for the
// butterflies).  Per token the angles pos * inv_freq are formed once, in
// binary64, one pair per thread, and their cosines and sines left in LDS for
// all heads.  A row is read a pass ahead of its turn.
//
// Bound: HBM.  16384 tokens of 64 heads of 128 take 97 to 114 us from card to card,
// 4.7 .. 5.5 TB/s, which is what a copy of as many bytes reaches; ragged prompts of up
// to 4099 tokens with 64 query and 8 cache heads 85 to 94.  A single token is its launch and five memory
// latencies, 3.7 us.
#include "paged.hpp"
#include "quant_math.hpp"

namespace quarot {
namespace {

// cos and sin of a (|a| < 2^31) rounded to binary32 once, from binary64:
// Cody-Waite reduction by k = rint(a 2/pi) with pi/2 in two parts (the first
// difference is exact: a and k hi are multiples of 2^-52 and the difference is
// below 1), then the Taylor sums to r^15 and r^16 on |r| <= pi/4, whose
// remainders are below 2^-54.  The angle of a position past 2^24 needs the 53
// bits; the polynomials cost one evaluation per token and pair.
__device__ __forceinline__ float2 cos_sin(double a)
{
    const double k = __builtin_rint(a * 0x1.45f306dc9c883p-1);
    double r = __builtin_fma(-k, 0x1.921fb54442d18p+0, a);
    r = __builtin_fma(-k, 0x1.1a62633145c07p-54, r);
    const double x = r * r;
    double s = -1.0 / 1307674368000.0;
    s = __builtin_fma(s, x, 1.0 / 6227020800.0);
    s = __builtin_fma(s, x, -1.0 / 39916800.0);
    s = __builtin_fma(s, x, 1.0 / 362880.0);
    s = __builtin_fma(s, x, -1.0 / 5040.0);
    s = __builtin_fma(s, x, 1.0 / 120.0);
    s = __builtin_fma(s, x, -1.0 / 6.0);
    s = __builtin_fma(s * x, r, r);
    double c = 1.0 / 20922789888000.0;
    c = __builtin_fma(c, x, -1.0 / 87178291200.0);
    c = __builtin_fma(c, x, 1.0 / 479001600.0);
    c = __builtin_fma(c, x, -1.0 / 3628800.0);
    c = __builtin_fma(c, x, 1.0 / 40320.0);
    c = __builtin_fma(c, x, -1.0 / 720.0);
    c = __builtin_fma(c, x, 1.0 / 24.0);
    c = __builtin_fma(c, x, -0.5);
    c = __builtin_fma(c, x, 1.0);
    const int q = (int)k;
    const float cf = (float)(q & 1 ? s : c), sf = (float)(q & 1 ? c : s);
    return make_float2((q + 1) & 2 ? -cf : cf, q & 2 ? -sf : sf);
}

constexpr int AP_THREADS = APPEND_THREADS;

// D elements a row; APPEND: keys and values go to the pages as well, and rows
// outside the sequences are left alone.
template <int D, bool APPEND>
__global__ __launch_bounds__(AP_THREADS) void k_rope_append(AppendArgs a)
{
    constexpr int L = D / 8;                 // lanes per row
    constexpr int LOGL = D == 64 ? 3 : D == 128 ? 4 : 5;
    constexpr int RPP = AP_THREADS / L;      // rows per pass
    __shared__ float2 cs[D / 2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t t = blockIdx.x;
    const int pos = lane_pos(lane) & (L - 1);

    // Row h of the token (the queries', keys', values' heads in turn), and for the
    // halves' pairs its other half.  A row is read a pass ahead, the first one
    // before anything is known of the token's sequence.
    const RopeArgs &ro = a.rope;
    const int heads = APPEND ? a.hq + 2 * a.hkv : a.hq, e0 = pos * 8;
    const bool in_rot = e0 < 2 * ro.half, low = e0 < ro.half;
    uint4 next, next_o = {};
    auto fetch = [&](int h) {
        const uint16_t *x = a.q + t * a.q_stride + h * D;
        if (APPEND && h >= a.hq)
            x = h >= a.hq + a.hkv ? a.v + t * a.v_stride + (h - a.hq - a.hkv) * D
                                  : a.k + t * a.k_stride + (h - a.hq) * D;
        next = *reinterpret_cast<const uint4 *>(x + e0);
        if (in_rot && !ro.interleaved && (!APPEND || h < a.hq + a.hkv))
            next_o = *reinterpret_cast<const uint4 *>(x + (low ? e0 + ro.half : e0 - ro.half));
    };
    const int h0 = blockIdx.y * RPP + tid / L;
    if (h0 < heads)
        fetch(h0);

    // the token's sequence and its slot in the pools (row of head 0, or -1)
    int at = (int)t;
    int64_t slot = -1;
    if constexpr (APPEND) {
        const PagedMap &m = a.map;
        int lo, n;
        search(m, lo, n, [&](int, int cu) { return cu <= (int)t; });
        const int bl = lo + min(lane, n - 1), c0 = m.cu[bl], c1 = m.cu[bl + 1], len = m.len[bl];
        const uint64_t mine = __ballot(c0 <= (int)t && (int)t < c1);
        if (mine == 0)
            return;
        const int i = __builtin_ctzll(mine), b = lo + i;
        at = (int)((uint32_t)__builtin_amdgcn_readlane(len, i) -
                   (uint32_t)(__builtin_amdgcn_readlane(c1, i) - (int)t));
        slot = pool_row(m, a.hkv, b, at);
    }

    if (tid < ro.half) {
        const int ax = (ro.axis[tid >> 4] >> (2 * (tid & 15))) & 3;
        const int p = ro.pos ? ro.pos[ax * ro.pos_stride + t] : at;
        cs[tid] = cos_sin((double)p * (double)ro.inv_freq[tid]);
    }
    __syncthreads();

    for (int h = h0; h < heads; h += gridDim.y * RPP) {
        const uint4 row_raw = next, other = next_o;
        if (h + (int)gridDim.y * RPP < heads)
            fetch(h + gridDim.y * RPP);
        const bool isq = h < a.hq, isv = APPEND && h >= a.hq + a.hkv;
        const int hh = isq ? h : isv ? h - a.hq - a.hkv : h - a.hq;
        if (!isq && slot < 0)
            continue;
        float v[8];
        unpack8(row_raw, v);
        if (!isv && in_rot) {
            if (ro.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float2 w = cs[(e0 + e) >> 1];
                    const float p = v[e], q = v[e + 1];
                    v[e] = p * w.x - q * w.y;
                    v[e + 1] = q * w.x + p * w.y;
                }
            } else {
                float o[8];
                unpack8(other, o);
                const float2 *w = cs + (low ? e0 : e0 - ro.half);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = v[e] * w[e].x, q = o[e] * w[e].y;
                    v[e] = low ? p - q : p + q;
                }
            }
        }
        if (isv ? a.rot_v : a.rot_k) {
#pragma unroll
            for (int s = 1; s < 8; s <<= 1)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(e & s)) {
                        const float p = v[e], q = v[e + s];
                        v[e] = p + q;
                        v[e + s] = p - q;
                    }
            const float sc = lane_stages<LOGL, 8>(v, lane, pos) * a.c;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = __builtin_fmaf(v[e], sc, 0.0f);  // a zero is +0
        }
        if (isq) {
            store8(a.qo + t * a.qo_stride + hh * D + e0, v);
            continue;
        }
        // quarot_kv_quant's scale, zero and codes of the group
        float mx = v[0], mn = v[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            mx = fmaxf(mx, v[e]);
            mn = fminf(mn, v[e]);
        }
        static_for<LOGL>([&](auto J) {
            if ((8 << J) < a.G) {
                mx = lane_max<J>(mx);
                mn = lane_min<J>(mn);
            }
        });
        // + 0: a bound that is a zero is +0
        const float mxc = (mx + 0.0f) * a.clip, mnc = (mn + 0.0f) * a.clip;
        const uint16_t s16 = f2h(div15(mxc - mnc)), z16 = f2h(mnc);
        const Divisor dv = make_divisor(h2f(s16));
        const float zf = h2f(z16);
        uint32_t pk = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            pk |= (asym_code_bits(v[e], dv, zf) & 15u) << (4 * e);
        const PagedPool &p = isv ? a.vp : a.kp;
        const int64_t row = slot + (int64_t)hh * a.map.page;
        *reinterpret_cast<uint32_t *>(p.c + row * (D / 2) + e0 / 2) = dv.ok ? pk : 0u;
        if (e0 % a.G == 0) {
            const int64_t gi = row * (D / a.G) + e0 / a.G;
            p.s[gi] = s16;
            p.z[gi] = z16;
        }
    }
}

template <int D>
hipError_t go(const AppendArgs &a, hipStream_t s)
{
    constexpr int RPP = AP_THREADS / (D / 8);
    const int heads = a.k ? a.hq + 2 * a.hkv : a.hq;
    const int passes = (heads + RPP - 1) / RPP;
    // few tokens: a block per pass of its heads (64 tokens of 80 rows 5.6 us, 8.6 with
    // a block each); many: a token per block, whose angles are formed once (16384 of
    // 64 rows 102 us, 143 with a block per pass)
    const int by = (int)std::min<int64_t>(passes, std::max<int64_t>(1, 2048 / a.map.T));
    const dim3 grid((unsigned)a.map.T, (unsigned)by);
    if (a.k)
        hipLaunchKernelGGL((k_rope_append<D, true>), grid, dim3(AP_THREADS), 0, s, a);
    else
        hipLaunchKernelGGL((k_rope_append<D, false>), grid, dim3(AP_THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t s)
{
    switch (a.D) {
    case 64: return go<64>(a, s);
    case 128: return go<128>(a, s);
    case 256: return go<256>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace quarot
