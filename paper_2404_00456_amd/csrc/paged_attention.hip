// Attention of new tokens over the paged 4-bit KV cache, for gfx950.
//
// Query i of sequence b sits at position p = len - n + i and sees the cached
// tokens t <= p with t > p - window (where there is a window) or t < sinks:
//   out = softmax_t(sm_scale q . khat_t) . vhat,  khat = code * scale + zero,
// and zero where it sees nothing.  The query heads of one cache head are rows
// of the same tile, so that a cached token is unpacked once for all of them:
// row r of a sequence is its new token r / rep, head r % rep.
//
// k_paged_tile: a block takes 32 rows per wave and walks over the tokens that
// any of them sees, 64 at a time.  The codes of a step become fp16 values in
// LDS (RN16 of code * scale + zero, one rounding, as quarot_kv_dequant gives
// them; half an fp16 step of a key or value is what the fp16 output keeps of
// it as well).  Scores are taken transposed, S = K Q^T, so that the lane that
// holds a query's scores also holds its share of the weights as the B operand
// of O = V^T P^T: the weights never leave their registers.  Softmax sums and
// outputs are binary32; weights are rounded to fp16 for the product.
#include <algorithm>

#include "lds_dma.hpp"
#include "paged.hpp"

namespace quarot {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 h2v __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int TT = paged::STEP;

// What a block of MR query rows works on.
struct Work : paged::Span {
    int b;     // sequence
    int tok0;  // first batch row (new token) of the sequence
};

template <int MR>
__device__ __forceinline__ Work find_work(const PagedAttnArgs &a, int slot, int *sh)
{
    const PagedMap &m = a.map;
    if (threadIdx.x == 0)
        *sh = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < m.B; b += blockDim.x)
        if (paged::first_slot((int64_t)m.cu[b] * a.rep, b, MR) <= slot &&
            slot < paged::first_slot((int64_t)m.cu[b + 1] * a.rep, b + 1, MR))
            *sh = b;
    __syncthreads();
    Work w = {};
    w.b = __builtin_amdgcn_readfirstlane(*sh);
    if (w.b < 0)
        return w;
    const int c0 = m.cu[w.b], c1 = m.cu[w.b + 1];
    static_cast<paged::Span &>(w) =
        paged::span(c0, c1, m.len[w.b], m.T, m.max_pages * m.page, a.rep,
                    slot - paged::first_slot((int64_t)c0 * a.rep, w.b, MR), MR, a.window, a.sinks,
                    a.splits, a.least);
    w.tok0 = c0;
    return w;
}

__device__ __forceinline__ h2v bits_h2(uint32_t b)
{
    return __builtin_bit_cast(h2v, b);
}

// Masks and exponents of the code pairs, in registers: v_and_or_b32 takes no
// literal, and with constants in sight the compiler splits it into an and and an
// or, so they pass through an empty asm once.
struct NibConst {
    uint32_t mlo, mhi, glo, ghi;
};

__device__ __forceinline__ NibConst nib_const()
{
    NibConst k = {0x000F000Fu, 0x00F000F0u, 0x64006400u, 0x54005400u};
    __asm__("" : "+s"(k.mlo), "+s"(k.mhi), "+v"(k.glo), "+v"(k.ghi));
    return k;
}

// Two codes as fp16 integers: or-ed into the significand of 1024 (where fp16
// values are spaced by 1) or, for the nibbles at bits 4-7 and 20-23, of 64
// (spaced by 1/16), minus that.
template <bool HI>
__device__ __forceinline__ h2v nib_pair(uint32_t w, const NibConst &k)
{
    const uint32_t x = HI ? (w & k.mhi) | k.ghi : (w & k.mlo) | k.glo;
    const _Float16 b = HI ? (_Float16)-64.0f : (_Float16)-1024.0f;
    const h2v off = {b, b};
    return bits_h2(x) + off;
}

__device__ __forceinline__ h2v pk_rtz(float a, float b)
{
    return __builtin_bit_cast(h2v, __builtin_amdgcn_cvt_pkrtz(a, b));
}

__device__ __forceinline__ h2v fma2(h2v a, h2v b, h2v c)
{
    return __builtin_elementwise_fma(a, b, c);
}

// 16 bytes of 8 fp16 elements in the order 0, 4, 1, 5, 2, 6, 3, 7, in which
// the nibble pairs of a dword of codes come out
__device__ __forceinline__ uint4 nib_order(uint4 r)
{
    return make_uint4(perm_b32(r.z, r.x, 0x05040100u), perm_b32(r.z, r.x, 0x07060302u),
                      perm_b32(r.w, r.y, 0x05040100u), perm_b32(r.w, r.y, 0x07060302u));
}

// The values of a dword of codes (8 elements) in that order.
__device__ __forceinline__ uint4 unpack8(uint32_t w, h2v s, h2v z, const NibConst &nk)
{
    const uint32_t w8 = w >> 8;
    return make_uint4(__builtin_bit_cast(uint32_t, fma2(nib_pair<false>(w, nk), s, z)),
                      __builtin_bit_cast(uint32_t, fma2(nib_pair<true>(w, nk), s, z)),
                      __builtin_bit_cast(uint32_t, fma2(nib_pair<false>(w8, nk), s, z)),
                      __builtin_bit_cast(uint32_t, fma2(nib_pair<true>(w8, nk), s, z)));
}

__device__ __forceinline__ h2v pair_of(uint32_t lo, uint32_t hi)
{
    return bits_h2(lo | (hi << 16));
}

// Token block i of a step: K as fp16 rows [64][D], the 16-byte unit u of row t
// at u ^ (t & swizzle); V transposed, [D][64] with the tokens of a 16-token
// group in the order that the scores' registers have (4 h + r, then 8 + 4 h +
// r, for lane half h), the 16-byte unit u of dimension d at u ^ ((d ^ d / 8) &
// 7).  Both swizzles spread the writes and the reads over the banks.
template <int D>
struct Stage {
    static constexpr int K_BYTES = TT * D * 2, V_BYTES = TT * D * 2;
    static constexpr int KSW = D == 64 ? 7 : 15;
    uint8_t k[K_BYTES];
    uint8_t v[V_BYTES];
    int ok[4];  // the page of each 16-token group exists
};

// What a thread stages of a step: a step is 2 D items of 32 elements of a key and
// 2 D items of 8 elements of 4 tokens' values.  With more than 2 D threads the
// waves part the kinds between them, so that one item a thread is in flight;
// otherwise each thread has N of both.
template <int D, int NT>
struct Share {
    static constexpr bool PART = NT > 2 * D;
    static constexpr int N = PART ? 1 : 2 * D / NT;
};

struct Item {
    int64_t row;   // pool row of the next read (its first token's), or -1
    int t;         // that token
    int ok;        // the page of what was read exists
    uint4 c;       // codes: a key's 32, or 8 of each of 4 tokens
    uint2 s, z;    // scales and zeros: a key's, or those of the four tokens
};

template <int D, int NT, bool KEY>
__device__ __forceinline__ void look_up(const PagedAttnArgs &a, const Work &w, int h, int t0, int i,
                                        Item &r)
{
    const int item = ((int)threadIdx.x + i * NT) & (2 * D - 1);
    r.t = t0 + (KEY ? item / (D / 32) : item / (D / 8) * 4);
    const int64_t row = pool_row(a.map, a.hkv, w.b, r.t);  // the next three too: pages are 16 n
    r.row = row >= 0 ? row + (int64_t)h * a.map.page : -1;
}

// Rows of no page are read as row 0 of the pool and take no part: a key by `ok`,
// values by constants of 0.
template <int D, int NT, bool KEY, bool ONE>
__device__ __forceinline__ void read_ahead(const PagedAttnArgs &a, const Work &w, int i, Item &r)
{
    const int ng = ONE ? 1 : D / a.G;
    const int item = ((int)threadIdx.x + i * NT) & (2 * D - 1);
    r.ok = r.row >= 0;
    const int64_t row = r.ok ? r.row : 0;
    if constexpr (KEY) {
        const int sl = item % (D / 32);
        const int64_t g = row * ng + (ONE ? 0 : sl * 32 / a.G);
        r.c = *reinterpret_cast<const uint4 *>(a.kp.c + row * (D / 2) + sl * 16);
        r.s.x = a.kp.s[g];
        r.z.x = a.kp.z[g];
    } else {
        const int dg = item % (D / 8);
        const uint8_t *src = a.vp.c + row * (D / 2) + dg * 4;
        r.c.x = *reinterpret_cast<const uint32_t *>(src);
        r.c.y = *reinterpret_cast<const uint32_t *>(src + D / 2);
        r.c.z = *reinterpret_cast<const uint32_t *>(src + D);
        r.c.w = *reinterpret_cast<const uint32_t *>(src + 3 * (D / 2));
        if constexpr (ONE) {  // four tokens' constants lie side by side
            r.s = *reinterpret_cast<const uint2 *>(a.vp.s + row);
            r.z = *reinterpret_cast<const uint2 *>(a.vp.z + row);
        } else {
            uint32_t s[4], z[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int64_t g = (row + x) * ng + dg * 8 / a.G;
                s[x] = a.vp.s[g];
                z[x] = a.vp.z[g];
            }
            r.s = make_uint2(s[0] | (s[1] << 16), s[2] | (s[3] << 16));
            r.z = make_uint2(z[0] | (z[1] << 16), z[2] | (z[3] << 16));
        }
        // tokens that no row sees take a weight of 0, and 0 times what a slot
        // holds that was never written may be NaN
        if (!(r.ok & (r.t + 4 <= w.hi) & (r.t >= w.low))) {
            uint32_t keep[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int t = r.t + x;
                keep[x] = (r.ok & (t < w.hi) & ((t >= w.low) | (t < a.sinks))) ? 0xFFFFu : 0u;
            }
            const uint32_t k01 = keep[0] | (keep[1] << 16), k23 = keep[2] | (keep[3] << 16);
            r.s = make_uint2(r.s.x & k01, r.s.y & k23);
            r.z = make_uint2(r.z.x & k01, r.z.y & k23);
        }
    }
}

template <int D, int NT, bool KEY>
__device__ __forceinline__ void put(Stage<D> &st, int i, const Item &r, const NibConst &nk)
{
    const int item = ((int)threadIdx.x + i * NT) & (2 * D - 1);
    if constexpr (KEY) {
        const int t = item / (D / 32), sl = item % (D / 32);
        const h2v s = bits_h2(perm_b32(r.s.x, r.s.x, 0x01000100u));
        const h2v z = bits_h2(perm_b32(r.z.x, r.z.x, 0x01000100u));
        const uint32_t w[4] = {r.c.x, r.c.y, r.c.z, r.c.w};
#pragma unroll
        for (int x = 0; x < 4; ++x)
            *reinterpret_cast<uint4 *>(st.k + t * (2 * D) + (((4 * sl + x) ^ (t & Stage<D>::KSW)) * 16)) =
                unpack8(w[x], s, z, nk);
        st.ok[t >> 4] = r.ok;  // (every lane of a 16-token group writes the same)
    } else {
        const int q = item / (D / 8), dg = item % (D / 8);
        // tokens 4 q .. 4 q + 3: 16-token group q / 4, lane half q % 2, 8-byte
        // piece (q / 2) % 2
        const int unit = (q >> 2) * 2 + (q & 1), piece = (q >> 1) & 1;
        const h2v s01 = bits_h2(r.s.x), s23 = bits_h2(r.s.y);
        const h2v z01 = bits_h2(r.z.x), z23 = bits_h2(r.z.y);
#pragma unroll
        for (int bt = 0; bt < 4; ++bt) {
            // byte bt of two tokens in bytes 0 and 2
            const uint32_t sel = (uint32_t)bt | 0x0C00u | ((uint32_t)(4 + bt) << 16) | 0x0C000000u;
            const uint32_t x01 = perm_b32(r.c.y, r.c.x, sel), x23 = perm_b32(r.c.w, r.c.z, sel);
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const int d = dg * 8 + 2 * bt + hi;
                const h2v a01 = hi ? nib_pair<true>(x01, nk) : nib_pair<false>(x01, nk);
                const h2v a23 = hi ? nib_pair<true>(x23, nk) : nib_pair<false>(x23, nk);
                *reinterpret_cast<uint2 *>(st.v + d * (2 * TT) + ((unit ^ ((d ^ (d >> 3)) & 7)) * 16) +
                                           piece * 8) =
                    make_uint2(__builtin_bit_cast(uint32_t, fma2(a01, s01, z01)),
                               __builtin_bit_cast(uint32_t, fma2(a23, s23, z23)));
            }
        }
    }
}

// Block id -> (slot, split, cache head): heads next to each other, so that
// with eight of them each XCD keeps to one head's cache; late slots (long
// rows of a prompt) first.
struct Place {
    int slot, split, h;
};

__device__ __forceinline__ Place place(const PagedAttnArgs &a, int slots)
{
    const uint32_t id = blockIdx.x;
    const uint32_t rest = id / (uint32_t)a.hkv;
    Place p;
    p.h = (int)(id % (uint32_t)a.hkv);
    p.split = (int)(rest % (uint32_t)a.splits);
    p.slot = slots - 1 - (int)(rest / (uint32_t)a.splits);
    return p;
}

// Orders within a step, for the scheduler: what a wave issues runs in order, so
// matrix products and vector instructions overlap only where they alternate.
__device__ __forceinline__ void mix_softmax()
{
#if 0
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
#endif
}

__device__ __forceinline__ void mix_stage()
{
}

template <int D, int NW, bool ONE>
__global__ __launch_bounds__(64 * NW) void k_paged_tile(PagedAttnArgs a, int slots)
{
    constexpr int NT = 64 * NW, MR = 32 * NW;
    constexpr int KS = D / 16, DB = D / 32;
    // stages: one that is multiplied, the next one, and one that is written while
    // some wave may still be at the first (two, and a barrier more, where three
    // do not fit)
    constexpr int NB = D == 256 ? 2 : 3;
    __shared__ __align__(16) Stage<D> st[NB];
    __shared__ int shb;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 31, hf = lane >> 5;
    const Place pl = place(a, slots);
    const Work w = find_work<MR>(a, pl.slot, &shb);
    if (w.rows == 0 || pl.split >= w.used)
        return;
    const float inf = __builtin_inff();
    const float c2 = a.sm_scale * 1.44269504088896340736f;  // log2(e)

    // this lane's query: row, batch row, head, position
    const int row = min(w.row0 + wave * 32 + n, w.rows - 1);
    const bool live = w.row0 + wave * 32 + n < w.rows;
    const int qi = row / a.rep;
    const int head = pl.h * a.rep + (row - qi * a.rep);
    const int p = w.pos0 + qi;
    const int64_t trow = w.tok0 + qi;
    const int wfirst = a.window > 0 ? p - a.window : -1;  // tokens up to here only as sinks
    v8h qb[KS];
    {
        const uint16_t *qr = a.q + trow * a.q_stride + (int64_t)head * D;
#pragma unroll
        for (int k = 0; k < KS; ++k)
            qb[k] = __builtin_bit_cast(
                v8h, nib_order(*reinterpret_cast<const uint4 *>(qr + 16 * k + 8 * hf)));
    }

    v16f o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[d][r] = 0.0f;
    float m = -inf, l = 0.0f;  // in log2 units; this lane's half of the sum

    const int begin = pl.split * w.per, end = min(w.steps, begin + w.per);
    auto token0 = [&](int i) { return paged::step_token(w, i < end ? i : end - 1); };
    const int pmin = w.pos0 + w.row0 / a.rep, pmax = w.pos0 + (min(w.row0 + MR, w.rows) - 1) / a.rep;

    // scores of the 32 tokens of half u: register r holds token
    // 32 u + 8 (r / 4) + 4 hf + r % 4
    auto score = [&](const Stage<D> &sg, int u) {
        v16f s;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = 0.0f;
        const int t = 32 * u + n;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const v8h kf = *reinterpret_cast<const v8h *>(
                sg.k + t * (2 * D) + (((2 * k + hf) ^ (t & Stage<D>::KSW)) * 16));
            s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qb[k], s, 0, 0, 0);
        }
        return s;
    };
    // their weights as the value product's B operands, and the sums
    auto weigh = [&](const v16f &s, v8h *pb, float ms) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -ms));
            sum[r & 3] += e;
            pb[r >> 3][r & 7] = (_Float16)e;
        }
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    };
    auto hide = [&](v16f &s, int t0, const int *ok, int u) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = t0 + 32 * u + 8 * (r >> 2) + 4 * hf + (r & 3);
            const bool see = (t <= p) & ((t > wfirst) | (t < a.sinks)) & (ok[2 * u + (r >> 3)] != 0);
            s[r] = see ? s[r] : -inf;
        }
    };
    // takes the weights' sum; where they pass what fp16 holds, or there is no
    // reference yet, the reference moves to the largest score
    auto settle = [&](const v16f &s, v8h *pb, float ls) {
        if (__builtin_expect(__any(!(ls <= 0x1p15f) | (m == -inf)), 0)) {
            float mt = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r)
                mt = fmaxf(mt, s[r]);
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt),
                                                             false, false);
            const float mn = fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2);
            const float ms = mn > -inf ? mn : 0.0f;  // nothing seen so far: weights 0
            const float f = m > -inf ? __builtin_amdgcn_exp2f(m - ms) : 0.0f;
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    o[d][r] *= f;
                    asm volatile("" : "+v"(o[d]));
                }
            ls = weigh(s, pb, ms);
        }
        l += ls;
    };
    auto add_values = [&](const Stage<D> &sg, int u, const v8h *pb) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int unit = (2 * u + x) * 2 + hf;
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int dim = 32 * d + n;
                const v8h vf = *reinterpret_cast<const v8h *>(
                    sg.v + dim * (2 * TT) + ((unit ^ ((dim ^ (dim >> 3)) & 7)) * 16));
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pb[x], o[d], 0, 0, 0);
            }
        }
    };

    if (begin < end) {
        using Sh = Share<D, NT>;
        const NibConst nk = nib_const();
        // 0: this wave stages keys, 1: values, 2: nothing
        const int role = Sh::PART ? __builtin_amdgcn_readfirstlane(tid / (2 * D)) : 0;
        Item kv[Sh::PART ? 1 : 2][Sh::N];
        // f(a kind of item, its items) for what this wave stages, then once `also`
        auto each = [&](auto f, auto also) {
            if constexpr (Sh::PART) {
                if (role == 0) {
                    f(std::true_type(), kv[0]);
                    also();
                } else if (NT <= 4 * D || role == 1) {
                    f(std::false_type(), kv[0]);
                    also();
                } else {
                    also();
                }
            } else {
                f(std::true_type(), kv[0]);
                f(std::false_type(), kv[1]);
                also();
            }
        };
        auto look = [&](int step) {
            return [&, step](auto key, Item *r) {
#pragma unroll
                for (int i = 0; i < Sh::N; ++i)
                    look_up<D, NT, decltype(key)::value>(a, w, pl.h, token0(step), i, r[i]);
            };
        };
        auto read = [&](auto key, Item *r) {
#pragma unroll
            for (int i = 0; i < Sh::N; ++i)
                read_ahead<D, NT, decltype(key)::value, ONE>(a, w, i, r[i]);
        };
        auto write = [&](Stage<D> &to) {
            return [&](auto key, Item *r) {
#pragma unroll
                for (int i = 0; i < Sh::N; ++i)
                    put<D, NT, decltype(key)::value>(to, i, r[i], nk);
            };
        };
        auto nothing = [] {};
        each(look(begin), nothing);
        each(read, nothing);
        each(write(st[0]), nothing);
        each(look(begin + 1), nothing);
        each(read, nothing);
        each(look(begin + 2), nothing);
        __syncthreads();
        v16f s0 = score(st[0], 0), s1;
        int cur = 0;
        for (int i = begin; i < end; ++i) {
            const int t0 = token0(i);
            const Stage<D> &sc = st[cur];
            const int nx = cur + 1 < NB ? cur + 1 : 0;
            const int ok[4] = {sc.ok[0], sc.ok[1], sc.ok[2], sc.ok[3]};
            const bool edge = !(ok[0] & ok[1] & ok[2] & ok[3]) || t0 + TT - 1 > pmin ||
                              (a.window > 0 && t0 <= pmax - a.window);
            v8h pb[2];
            if (edge)
                hide(s0, t0, ok, 0);
            s1 = score(sc, 1);
            float ls = weigh(s0, pb, m > -inf ? m : 0.0f);
            mix_softmax();
            settle(s0, pb, ls);
            each(
                [&](auto key, Item *r) {
                    write(st[nx])(key, r);
                    read(key, r);
                    look(i + 3)(key, r);
                },
                nothing);
            add_values(sc, 0, pb);
            if (edge)
                hide(s1, t0, ok, 1);
            __syncthreads();  // the next step's stage is whole
            s0 = score(st[nx], 0);
            ls = weigh(s1, pb, m > -inf ? m : 0.0f);
            mix_softmax();
            settle(s1, pb, ls);
            add_values(sc, 1, pb);
            if constexpr (NB == 2)
                __syncthreads();  // this one may be overwritten
            cur = nx;
        }
    }

    {
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false,
                                                         false);
        l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    if (!live)
        return;
    if (w.used == 1) {
        const float f = l > 0.0f ? 1.0f / l : 0.0f;
        uint16_t *dst = a.out + trow * a.out_stride + (int64_t)head * D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                uint2 v;
                v.x = (uint32_t)f2h(o[d][r] * f) | ((uint32_t)f2h(o[d][r + 1] * f) << 16);
                v.y = (uint32_t)f2h(o[d][r + 2] * f) | ((uint32_t)f2h(o[d][r + 3] * f) << 16);
                *reinterpret_cast<uint2 *>(dst + 32 * d + 2 * r + 4 * hf) = v;
            }
    } else {
        const int64_t pr = (trow * a.hq + head) * a.splits + pl.split;
        float *dst = a.part_o + pr * D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(dst + 32 * d + 2 * r + 4 * hf) =
                    make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
        if (hf == 0)
            *reinterpret_cast<float2 *>(a.part_ml + 2 * pr) = make_float2(m, l);
    }
}

// ---- few query rows: single tokens, and a few that were guessed ahead -------
//
// k_paged_rows: up to 16 query rows (new tokens times the heads of a cache head)
// of a sequence, one group per cached row.  Four waves take the block's token
// blocks of 64 in turn, straight from memory to registers, 16 tokens at a time
// as in the dense decode kernels: A = the K codes as fp16 integers against B =
// the queries, then A = the weights against B = the V codes.  Codes enter as
// they are, so that nothing of a key or value is rounded:
//   q . khat_t = ks_t (q . code_t) + kz_t sum(q),
//   sum_t p_t vhat_t = sum_t (p_t vs_t) code_t + sum_t p_t vz_t.
// A code c is or-ed into an fp16 significand: as 64 + c in the K operand, whose
// offset 64 sum(q) is taken off by the scores' initial accumulator (6 of
// binary32's 24 bits of scores that are far below it anyway), and as 1024 + c or
// 64 + c in the V operand, taken off by a packed add: an output over many tokens
// is small beside the sum of its weights, and offsets of 128 left in the
// products cost half an fp16 step over 32768 tokens.
//
// The weights p_t vs_t are two fp16 parts, an A operand each, 22 bits together
// while they are above 2^-14.  So the reference m that is taken off the scores x
// (log2 units) follows the weights and not the scores: it makes the first step's
// largest weight 1 whatever the values' scale is, and moves when a weight passes
// 2^15.  (Scales below 2^-24, none but 0 in fp16, count as that, so that rows of
// equal values have a reference.)
//
// A wave's codes and constants come through a ring of its own in LDS, 32 tokens
// a stage, by loads that go from memory straight there (16 bytes a lane): the
// next stage is on its way while this one is multiplied, at no registers, and
// the lanes take each cached row in the pieces that the matrix operands want.
constexpr int ROWS_W = 4;   // waves of a block
constexpr int ROWS_NS = 2;  // stages of a wave's ring

template <int D>
struct RowsRing {
    static constexpr int KB = 32 * D / 2;  // bytes of a stage's K codes, and of its V codes
    static constexpr int STAGE = 2 * KB + 256;  // and ks, kz, vs, vz of 32 tokens
    static constexpr int LOADS = 2 * (KB / 1024) + 1;
    static constexpr int UPR = D / 32;  // 16-byte units of a row
    // K: unit c of row n at c ^ swz(n), so that 16 rows' same unit falls on
    // different banks
    __device__ static int swz(int n)
    {
        return D == 128 ? (n >> 2) & 3 : D == 256 ? (n >> 1) & 7 : 0;
    }
    // V: token 4 g + j of a 16-token group is row 4 j + g, so that the four lane
    // groups' rows lie side by side
    __device__ static int token_of(int r)
    {
        return 4 * (r & 3) + (r >> 2);
    }
};

template <int D>
__global__ __launch_bounds__(64 * ROWS_W)
    __attribute__((amdgpu_waves_per_eu(D == 256 ? 2 : 4, D == 256 ? 2 : 4))) void k_paged_rows(PagedAttnArgs a, int slots)
{
    using Ring = RowsRing<D>;
    constexpr int MR = paged::FEW_ROWS;
    constexpr int KW = D / 32;  // dwords of K codes of a lane: D / 4 elements of a token
    constexpr int VD = D / 16;  // dimensions of a lane in the value product
    constexpr int RED = ROWS_W * MR * (D + 2) * 4, RING = ROWS_W * ROWS_NS * Ring::STAGE;
    __shared__ __align__(16) uint8_t lds[RED > RING ? RED : RING];
    __shared__ int shb;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 15, g = lane >> 4;
    const Place pl = place(a, slots);
    const Work w = find_work<MR>(a, pl.slot, &shb);
    if (w.rows == 0 || pl.split >= w.used)
        return;
    const float inf = __builtin_inff();
    const float c2 = a.sm_scale * 1.44269504088896340736f;  // log2(e)
    const int R = min(MR, w.rows - w.row0);

    // this lane's query (column n of the scores)
    const int row = w.row0 + min(n, R - 1), qi = row / a.rep;
    const int p = w.pos0 + qi;
    const int wfirst = a.window > 0 ? p - a.window : -1;
    const int pmin = w.pos0 + w.row0 / a.rep, pmax = w.pos0 + (w.row0 + R - 1) / a.rep;
    v8h qb[KW];
    float qsum = 0.0f;
    {
        const uint16_t *qr = a.q + (int64_t)(w.tok0 + qi) * a.q_stride +
                             (int64_t)(pl.h * a.rep + (row - qi * a.rep)) * D + (D / 4) * g;
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            qb[k] = __builtin_bit_cast(v8h, nib_order(*reinterpret_cast<const uint4 *>(qr + 8 * k)));
#pragma unroll
            for (int e = 0; e < 8; ++e)
                qsum += (float)qb[k][e];
        }
        float2 t = lane_pair_swap<4>(qsum);
        qsum = t.x + t.y;
        t = lane_pair_swap<5>(qsum);
        qsum = t.x + t.y;
    }
    const float qs = qsum * c2, q64 = -64.0f * qsum;

    v4f o[VD];
#pragma unroll
    for (int d = 0; d < VD; ++d)
        o[d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -inf, l = 0.0f, zs = 0.0f;

    // this wave's stages: stage k is half k % 2 of step begin + wave + 4 (k / 2)
    const int begin = pl.split * w.per + wave, end = min(w.steps, pl.split * w.per + w.per);
    const int stages = begin < end ? 2 * ((end - begin + ROWS_W - 1) / ROWS_W) : 0;
    auto token_at = [&](int k) {
        return paged::step_token(w, begin + (k >> 1) * ROWS_W) + 32 * (k & 1);
    };
    uint8_t *ring = lds + wave * (ROWS_NS * Ring::STAGE);
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(
        (uint32_t)reinterpret_cast<uintptr_t>(
            (__attribute__((address_space(3))) uint8_t *)ring));

    // this lane's source within a 16-token group (a load of K or V codes is 1024
    // / D * 2 tokens), and its constants' array
    constexpr int TPL = 2048 / D;  // tokens of a load: 32, 16, 8
    uint32_t koff[TPL < 16 ? 2 : 1], voff[TPL < 16 ? 2 : 1];
#pragma unroll
    for (int x = 0; x < (TPL < 16 ? 2 : 1); ++x) {
        const int rw = (x * TPL + lane / Ring::UPR) & 15, c = lane % Ring::UPR;
        koff[x] = rw * (D / 2) + (c ^ Ring::swz(rw)) * 16;
        voff[x] = Ring::token_of(rw) * (D / 2) + c * 16;
    }
    const uint16_t *carr = lane < 16 ? a.kp.s : lane < 32 ? a.kp.z : lane < 48 ? a.vp.s : a.vp.z;
    carr += (lane & 7) * 2;

    int64_t base = -1;  // pool rows of the next 64 groups of 16 tokens, one a lane
    auto issue = [&](int k) -> int {
        if ((k & 31) == 0) {
            const int kk = k + (lane >> 1);
            base = -1;
            if (kk < stages) {
                const int t = token_at(kk) + 16 * (lane & 1);
                if (t < w.hi)
                    base = pool_row(a.map, a.hkv, w.b, t);
                if (base >= 0)
                    base += (int64_t)pl.h * a.map.page;
            }
        }
        int64_t r0[2];
        int ok = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int src = 2 * (k & 31) + u;
            const uint32_t blo = __builtin_amdgcn_readlane((uint32_t)base, src);
            const uint32_t bhi = __builtin_amdgcn_readlane((uint32_t)(base >> 32), src);
            r0[u] = (int64_t)(((uint64_t)bhi << 32) | blo);
            ok |= r0[u] >= 0 ? 1 << u : 0;
            r0[u] = r0[u] >= 0 ? r0[u] : 0;  // a row of the pool, masked where it is used
        }
        const uint32_t at = ring_at + (uint32_t)(k % ROWS_NS) * Ring::STAGE;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage's last reads
        if constexpr (D == 64) {
            const int64_t rl = (lane >= 32 ? r0[1] : r0[0]) * (D / 2);
            dma16(a.kp.c + rl + koff[0], at);
            dma16(a.vp.c + rl + voff[0], at + Ring::KB);
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < 16 / TPL; ++x) {
                    dma16s(koff[x], a.kp.c + r0[u] * (D / 2), at + (u * (16 / TPL) + x) * 1024);
                    dma16s(voff[x], a.vp.c + r0[u] * (D / 2),
                           at + Ring::KB + (u * (16 / TPL) + x) * 1024);
                }
        }
        dma4(carr + (lane & 8 ? r0[1] : r0[0]), at + 2 * Ring::KB);
        return ok;
    };

    const NibConst nk = nib_const();
    int ok_next = stages > 0 ? issue(0) : 0;
    for (int k = 0; k < stages; ++k) {
        const int ok = ok_next, th = token_at(k);
        if (k + 1 < stages) {
            ok_next = issue(k + 1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Ring::LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const uint8_t *stg = ring + (k % ROWS_NS) * Ring::STAGE;
        const uint8_t *cst = stg + 2 * Ring::KB + 8 * g;  // + 64 array + 32 group
        float x[2][4];
        _Float16 ksh[2][4], kzh[2][4], vsh[2][4], vzh[2][4];  // enter v_fma_mix as they are
        auto halfs = [&](int arr, int u, _Float16 *f) {
            const uint2 v = *reinterpret_cast<const uint2 *>(cst + 64 * arr + 32 * u);
            const h2v lo = bits_h2(v.x), hi = bits_h2(v.y);
            f[0] = lo[0];
            f[1] = lo[1];
            f[2] = hi[0];
            f[3] = hi[1];
        };
        const float ms = m > -inf ? m : 0.0f;  // nothing seen so far: weights 0
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t kc[KW];
            {
                const uint8_t *kr = stg + u * (Ring::KB / 2) + n * (D / 2);
                if constexpr (D == 64) {
                    __builtin_memcpy(kc, __builtin_assume_aligned(kr + 8 * g, 8), 8);
                } else {
#pragma unroll
                    for (int c = 0; c < KW / 4; ++c)
                        __builtin_memcpy(kc + 4 * c,
                                         __builtin_assume_aligned(
                                             kr + (((KW / 4) * g + c) ^ Ring::swz(n)) * 16, 16), 16);
                }
            }
            v4f acc = {q64, q64, q64, q64};
#pragma unroll
            for (int c = 0; c < KW; ++c) {
                const uint32_t wd = kc[c];
                auto f64 = [&](uint32_t b) { return (b & nk.mhi) | nk.ghi; };
                const uint4 kf = make_uint4(f64(wd << 4), f64(wd), f64(wd >> 4), f64(wd >> 8));
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, kf), qb[c], acc,
                                                             0, 0, 0);
            }
            halfs(0, u, ksh[u]);
            halfs(1, u, kzh[u]);
            halfs(2, u, vsh[u]);
            halfs(3, u, vzh[u]);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                x[u][r] = __builtin_fmaf((float)ksh[u][r], acc[r] * c2,
                                         __builtin_fmaf((float)kzh[u][r], qs, -ms));
        }
        if (ok != 3 || th + 31 > pmin || (a.window > 0 && th <= pmax - a.window)) {
            asm volatile("");  // a branch, not selects in every step
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = th + 16 * u + 4 * g + r;
                    const bool see = (ok >> u & 1) && t <= p && (t > wfirst || t < a.sinks);
                    x[u][r] = see ? x[u][r] : -inf;
                    // a weight of 0 times what a slot that was never written
                    // holds may be NaN
                    vsh[u][r] = see ? vsh[u][r] : (_Float16)0.0f;
                    vzh[u][r] = see ? vzh[u][r] : (_Float16)0.0f;
                }
        }
        // weights, sums, and whether the reference still does
        float wt[2][4], ln = l, zn = zs, most = 0.0f;
        auto weigh = [&]() {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f(x[u][r]);
                    ln += e;
                    zn = __builtin_fmaf(e, (float)vzh[u][r], zn);
                    wt[u][r] = __builtin_fmaf(e, (float)vsh[u][r], 0.0f);
                    most = fmaxf(most, wt[u][r]);
                }
        };
        weigh();
        // (the sum as well: a value scale of 0 has no weight)
        if (__any(!(most <= 0x1p15f) || !(ln < 0x1p60f) || m == -inf)) {
            float y = -inf;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    y = fmaxf(y, x[u][r] + __builtin_amdgcn_logf(fmaxf((float)vsh[u][r], 0x1p-24f)));
            y = lane_max<4>(y);
            y = lane_max<5>(y);
            const float mn = fmaxf(m, ms + y);
            const float up = (mn > -inf ? mn : 0.0f) - ms;
            const float f = m > -inf ? __builtin_amdgcn_exp2f(-up) : 0.0f;
            m = mn;
            ln = l * f;
            zn = zs * f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[u][r] -= up;
            float fr[4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
                fr[r] = __shfl(f, 4 * g + r);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int d = 0; d < VD; ++d)
                    o[d][r] *= fr[r];
            weigh();
        }
        l = ln;
        zs = zn;
        uint32_t hh[4], ll[4];  // weights of the 32 tokens, as fp16 pairs
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                // the first part truncated, the second what that leaves
                const h2v hi = pk_rtz(wt[u][r], wt[u][r + 1]);
                hh[2 * u + r / 2] = __builtin_bit_cast(uint32_t, hi);
                ll[2 * u + r / 2] = __builtin_bit_cast(
                    uint32_t, pk_rtz(__builtin_fmaf((float)hi[0], -1.0f, wt[u][r]),
                                     __builtin_fmaf((float)hi[1], -1.0f, wt[u][r + 1])));
            }
        const v8h wh = __builtin_bit_cast(v8h, make_uint4(hh[0], hh[1], hh[2], hh[3]));
        const v8h wl = __builtin_bit_cast(v8h, make_uint4(ll[0], ll[1], ll[2], ll[3]));
        uint32_t vc[2][4][(VD + 7) / 8];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint8_t *vr = stg + Ring::KB + u * (Ring::KB / 2) + (4 * j + g) * (D / 2) +
                                    n * (D / 32);
                if constexpr (D == 64)
                    vc[u][j][0] = *reinterpret_cast<const uint16_t *>(vr);
                else
                    __builtin_memcpy(vc[u][j], __builtin_assume_aligned(vr, D / 32), D / 32);
            }
#pragma unroll
        for (int bt = 0; bt < VD / 2; ++bt) {
            // byte bt of tokens 4 g, 4 g + 1 (and + 2, + 3) of both groups
            const int wd = bt / 4;
            const uint32_t sel =
                (uint32_t)(bt & 3) | 0x0C00u | ((uint32_t)(4 + (bt & 3)) << 16) | 0x0C000000u;
            h2v lo[4], hi[4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const uint32_t b2 = perm_b32(vc[u][2 * t + 1][wd], vc[u][2 * t][wd], sel);
                    lo[2 * u + t] = nib_pair<false>(b2, nk);
                    hi[2 * u + t] = nib_pair<true>(b2, nk);
                }
            const v8h vlo = {lo[0][0], lo[0][1], lo[1][0], lo[1][1],
                             lo[2][0], lo[2][1], lo[3][0], lo[3][1]};
            const v8h vhi = {hi[0][0], hi[0][1], hi[1][0], hi[1][1],
                             hi[2][0], hi[2][1], hi[3][0], hi[3][1]};
            o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, vlo, o[2 * bt], 0, 0, 0);
            o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl, vlo, o[2 * bt], 0, 0, 0);
            o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, vhi, o[2 * bt + 1], 0, 0, 0);
            o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl, vhi, o[2 * bt + 1], 0, 0, 0);
        }
    }

    // each wave's (reference, sum, output) of its rows in LDS, then one of all
    {
        float2 t = lane_pair_swap<4>(l);
        l = t.x + t.y;
        t = lane_pair_swap<5>(l);
        l = t.x + t.y;
        t = lane_pair_swap<4>(zs);
        zs = t.x + t.y;
        t = lane_pair_swap<5>(zs);
        zs = t.x + t.y;
    }
    __syncthreads();  // every wave is through with its ring
    float (*red)[MR][D + 2] = reinterpret_cast<float (*)[MR][D + 2]>(lds);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float z = __shfl(zs, 4 * g + r);
#pragma unroll
        for (int d = 0; d < VD; ++d)
            red[wave][4 * g + r][VD * n + d] = o[d][r] + z;
    }
    if (g == 0) {
        red[wave][n][D] = m;
        red[wave][n][D + 1] = l;
    }
    __syncthreads();
    for (int i = tid; i < R * (D / 2); i += 64 * ROWS_W) {
        const int r = i / (D / 2), d = 2 * (i % (D / 2));
        float mx = -inf;
#pragma unroll
        for (int v = 0; v < ROWS_W; ++v)
            mx = fmaxf(mx, red[v][r][D]);
        const float ms = mx > -inf ? mx : 0.0f;
        float lt = 0.0f, oa = 0.0f, ob = 0.0f;
#pragma unroll
        for (int v = 0; v < ROWS_W; ++v) {
            const float f = __builtin_amdgcn_exp2f(red[v][r][D] - ms);
            lt = __builtin_fmaf(red[v][r][D + 1], f, lt);
            oa = __builtin_fmaf(red[v][r][d], f, oa);
            ob = __builtin_fmaf(red[v][r][d + 1], f, ob);
        }
        const int rr = w.row0 + r, ti = rr / a.rep;
        const int64_t trow = w.tok0 + ti;
        const int head = pl.h * a.rep + (rr - ti * a.rep);
        if (w.used == 1) {
            const float f = lt > 0.0f ? 1.0f / lt : 0.0f;
            *reinterpret_cast<uint32_t *>(a.out + trow * a.out_stride + (int64_t)head * D + d) =
                (uint32_t)f2h(oa * f) | ((uint32_t)f2h(ob * f) << 16);
        } else {
            const int64_t pr = (trow * a.hq + head) * a.splits + pl.split;
            *reinterpret_cast<float2 *>(a.part_o + pr * D + d) = make_float2(oa, ob);
            if (d == 0)
                *reinterpret_cast<float2 *>(a.part_ml + 2 * pr) = make_float2(mx, lt);
        }
    }
}

// The rows of a block whose splits were more than one.  WPR waves share a row's
// splits: one where there are few of them, four where one after the other they
// would cost a memory latency each.
template <int D, int MR, int WPR>
__global__ __launch_bounds__(256) void k_paged_combine(PagedAttnArgs a)
{
    constexpr int E = D / 64;  // elements of a lane
    constexpr int RPB = 4 / WPR;
    __shared__ int shb;
    __shared__ float red[WPR > 1 ? 4 : 1][D + 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = (int)(blockIdx.x % (uint32_t)a.hkv);
    const Work w = find_work<MR>(a, (int)(blockIdx.x / (uint32_t)a.hkv), &shb);
    if (w.rows == 0 || w.used == 1)
        return;
    const float inf = __builtin_inff();
    for (int r0 = blockIdx.y * RPB; r0 < MR && w.row0 + r0 < w.rows; r0 += gridDim.y * RPB) {
        const int r = r0 + wave / WPR, row = min(w.row0 + r, w.rows - 1), qi = row / a.rep;
        const bool live = r < MR && w.row0 + r < w.rows;
        const int head = h * a.rep + (row - qi * a.rep);
        const int64_t trow = w.tok0 + qi;
        const int64_t pr = (trow * a.hq + head) * a.splits;
        float mx = -inf;
        for (int s = lane; s < w.used; s += 64)
            mx = fmaxf(mx, a.part_ml[2 * (pr + s)]);
        static_for<6>([&](auto J) { mx = lane_max<J>(mx); });
        const float ms = mx > -inf ? mx : 0.0f;
        float l = 0.0f, o[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] = 0.0f;
#pragma unroll 8
        for (int s = wave % WPR; s < w.used; s += WPR) {
            const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (pr + s));
            const float f = __builtin_amdgcn_exp2f(ml.x - ms);  // 0 where it saw nothing
            l = __builtin_fmaf(ml.y, f, l);
            const float *src = a.part_o + (pr + s) * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e)
                o[e] = __builtin_fmaf(src[e], f, o[e]);
        }
        if constexpr (WPR > 1) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                red[wave][lane * E + e] = o[e];
            if (lane == 0)
                red[wave][D] = l;
            __syncthreads();
            l = red[0][D] + red[1][D] + red[2][D] + red[3][D];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = lane * E + e;
                o[e] = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
            }
            __syncthreads();
        }
        if (live && wave % WPR == 0) {
            const float f = l > 0.0f ? 1.0f / l : 0.0f;
            uint16_t *dst = a.out + trow * a.out_stride + (int64_t)head * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e)
                dst[e] = f2h(o[e] * f);
        }
    }
}

template <int D, int MR>
hipError_t go_combine(const PagedAttnArgs &a, int slots, hipStream_t s)
{
    const unsigned x = (unsigned)(slots * a.hkv);
    if (a.splits > 8)
        hipLaunchKernelGGL((k_paged_combine<D, MR, 4>), dim3(x, (unsigned)std::min(MR, a.rep * 4)),
                           dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((k_paged_combine<D, MR, 1>), dim3(x, (unsigned)std::max(1, MR / 32)),
                           dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D, int NW>
hipError_t go_tile(const PagedAttnArgs &a, hipStream_t s)
{
    constexpr int MR = 32 * NW;
    const int slots = (int)paged::slots(a.map.T, a.map.B, a.rep, MR);
    const dim3 grid((unsigned)((int64_t)slots * a.hkv * a.splits));
    if (a.G == D)
        hipLaunchKernelGGL((k_paged_tile<D, NW, true>), grid, dim3(64 * NW), 0, s, a, slots);
    else
        hipLaunchKernelGGL((k_paged_tile<D, NW, false>), grid, dim3(64 * NW), 0, s, a, slots);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1)
        return e;
    return go_combine<D, MR>(a, slots, s);
}

template <int D>
hipError_t go_few(const PagedAttnArgs &a, hipStream_t s)
{
    constexpr int MR = paged::FEW_ROWS;
    const int slots = (int)paged::slots(a.map.T, a.map.B, a.rep, MR);
    const dim3 grid((unsigned)((int64_t)slots * a.hkv * a.splits));
    hipLaunchKernelGGL((k_paged_rows<D>), grid, dim3(64 * ROWS_W), 0, s, a, slots);
    hipError_t e = hipGetLastError();
    return e != hipSuccess || a.splits == 1 ? e : go_combine<D, MR>(a, slots, s);
}

template <int D>
hipError_t go_rows(const PagedAttnArgs &a, int rows, hipStream_t s)
{
    if (rows == paged::FEW_ROWS)
        return go_few<D>(a, s);
    if constexpr (D < 256) {
        if (rows == 64)
            return go_tile<D, 2>(a, s);
        if (rows == 256)
            return go_tile<D, 8>(a, s);
    }
    return rows == 128 ? go_tile<D, 4>(a, s) : hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_paged_attention(const PagedAttnArgs &a, const paged::Plan &p, hipStream_t s)
{
    switch (a.D) {
    case 64: return go_rows<64>(a, p.rows, s);
    case 128: return go_rows<128>(a, p.rows, s);
    case 256: return go_rows<256>(a, p.rows, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace quarot
