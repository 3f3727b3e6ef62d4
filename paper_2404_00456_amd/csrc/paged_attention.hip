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
// them), once for all waves.  Scores are taken transposed, S = K Q^T, so that
// the lane that holds a query's scores also holds its share of the weights as the
// B operand of O = V^T P^T: the weights never leave their registers.  Softmax
// sums and outputs are binary32.  Three roundings to fp16 come on top of the
// output's own: keys, values, and weights for their product.  Each is off by half
// a step at most (a weight, where that is less, by 2^-31 of the row's largest) and at
// random, so that an output of many tokens is off by about
// 5e-4 of its size instead of 2e-4; taking the codes as they are and the weights
// in two parts, as k_paged_rows does, would be half as many matrix products again
// where these are what bounds the kernel.
//
// What bounds it: 32 rows by 32 tokens by 128 dimensions are 16 matrix
// instructions of 32 cycles, about 120 vector instructions (softmax 60, staging
// 40) and 18 KB of LDS traffic, each about half of a SIMD's time when two waves
// share it, so all three have to run beside each other.  8192 tokens of 64 heads
// on 8 take 1.18 to 1.24 ms from card to card, 890 .. 930 TFLOP/s where a
// library product of 8192^3 reaches 1330.  One wave with 64 rows a SIMD (half the
// LDS reads) was slower, 1.78 ms: its 512 registers are half accumulators, and
// the softmax works through copies of them.
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


// Log2 of a row's largest weight when its softmax reference is taken.  fp16's smallest
// numbers, and so the error of small weights, are as far below it as they can be; but
// the reference moves when weights pass 2^15, and nearer to that it does so more often
// (a prompt of 8192: 1212 us at 0, 1218 at 6, 1229 at 8; single tokens the same for 0
// and 8, a twentieth more for 12).
constexpr float TOP_TILE = 6.0f, TOP_ROWS = 8.0f;

// What a block of MR query rows works on.
struct Work : paged::Span {
    int b;     // sequence
    int tok0;  // first batch row (new token) of the sequence
};

__device__ __forceinline__ Work make_work(const PagedAttnArgs &a, int b, int c0, int c1, int len,
                                          int64_t block, int mr)
{
    Work w = {};
    w.b = b;
    w.tok0 = c0;
    static_cast<paged::Span &>(w) = paged::span(c0, c1, len, a.map.T, a.map.max_pages * a.map.page, a.rep,
                                                block, mr, a.window, a.sinks, a.splits, a.least);
    return w;
}

// Tiles: the sequence that has block row `slot`, from the lane that holds it.
template <int MR>
__device__ __forceinline__ Work find_work(const PagedAttnArgs &a, int slot)
{
    const PagedMap &m = a.map;
    int lo, n;
    search(m, lo, n, [&](int b, int cu) { return paged::first_slot((int64_t)cu * a.rep, b, MR) <= slot; });
    const int b = lo + min((int)threadIdx.x & 63, n - 1);
    const int c0 = m.cu[b], c1 = m.cu[b + 1], len = m.len[b];
    const uint64_t mine = __ballot(paged::first_slot((int64_t)c0 * a.rep, b, MR) <= slot &&
                                   slot < paged::first_slot((int64_t)c1 * a.rep, b + 1, MR));
    if (mine == 0)
        return Work{};
    const int i = __builtin_ctzll(mine), t0 = __builtin_amdgcn_readlane(c0, i);
    Work w = make_work(a, lo + i, t0, __builtin_amdgcn_readlane(c1, i), __builtin_amdgcn_readlane(len, i),
                       slot - paged::first_slot((int64_t)t0 * a.rep, lo + i, MR), MR);
    if (a.which == paged::MANY && w.rows <= paged::FEW_ROWS)
        w.rows = 0;
    return w;
}

// Few rows: slots 0 .. B - 1 are the sequences' first row blocks.  The further ones
// of sequences of more than 16 rows lie behind them, those of sequence b from slot
// B + (rows before b) / 16 on: no more than rows / 16 of them, so that they fit up
// to where those of b + 1 begin.
__device__ __forceinline__ Work few_work(const PagedAttnArgs &a, int slot)
{
    constexpr int MR = paged::FEW_ROWS;
    const PagedMap &m = a.map;
    int b = slot, extra = slot - m.B;
    int64_t rb = 0;
    if (extra >= 0) {
        int lo, n;
        search(m, lo, n, [&](int, int cu) { return (int64_t)cu * a.rep / MR <= extra; });
        const int64_t rows = (int64_t)m.cu[lo + min((int)threadIdx.x & 63, n - 1)] * a.rep;
        const uint64_t below = __ballot(((int)threadIdx.x & 63) < n && rows / MR <= extra);
        if (below == 0)
            return Work{};
        b = lo + 63 - __builtin_clzll(below);
        rb = 1 + extra - (int64_t)m.cu[b] * a.rep / MR;
    }
    const int c0 = m.cu[b], c1 = m.cu[b + 1];
    if (a.which == paged::FEW && ((int64_t)c1 - c0) * a.rep > MR)
        return Work{};
    return make_work(a, b, c0, c1, m.len[b], rb, MR);
}

// First partial result of a row.
__device__ __forceinline__ int64_t part_of(const PagedAttnArgs &a, const Work &w, int row, int h)
{
    return ((paged::part_row(a.which, w.b, w.tok0, a.rep) + row) * a.hkv + h) * a.splits;
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

// Two scale and zero pairs: bit 15 of the half of those under which some code would
// not be a finite fp16 value (code * s + z lies between z and 15 s + z, and so does
// its rounding; an exponent of all ones carries there).
__device__ __forceinline__ uint32_t spoils(uint32_t s, uint32_t z)
{
    const h2v fifteen = {(_Float16)15.0f, (_Float16)15.0f};
    const uint32_t b = __builtin_bit_cast(uint32_t, fma2(bits_h2(s), fifteen, bits_h2(z)));
    return ((b & 0x7FFF7FFFu) + 0x04000400u) & 0x80008000u;
}

// 16 bytes of 8 fp16 elements in the order 0, 4, 1, 5, 2, 6, 3, 7, in which
// the nibble pairs of a dword of codes come out
__device__ __forceinline__ uint4 nib_order(uint4 r)
{
    return make_uint4(perm_b32(r.z, r.x, 0x05040100u), perm_b32(r.z, r.x, 0x07060302u),
                      perm_b32(r.w, r.y, 0x05040100u), perm_b32(r.w, r.y, 0x07060302u));
}

// TS tokens in LDS.  K as fp16 rows [TS][D], with 16 bytes of padding, so that 16
// rows' same 16-byte unit falls on different banks and every address of a lane is
// one of its own and a constant.  V transposed, [D][TS], a dimension's tokens in
// the order that the scores' registers have (of a 16-token group 4 h + r, then
// 8 + 4 h + r, for lane half h: unit 2 group + h).  Rows of V change places in
// pairs and units within their row, so that neither the reads (16 bytes of
// neighbouring dimensions) nor the writes (8 bytes of every DV-th) meet on a bank;
// from one block of 32 dimensions to the next the units' order changes by one bit,
// so that two addresses of a lane do for all of them.
template <int D, int TS>
struct Stage {
    static constexpr int KP = 2 * D + 16, VP = 2 * TS;  // row pitches
    uint8_t k[TS * KP];
    uint8_t v[D * VP];
    int ok[TS / 16];  // the page of each 16-token group exists

    __device__ static int vrow(int d)
    {
        return (d ^ (((d >> 2) ^ (d >> 3)) & 1)) * VP;
    }
    __device__ static int vunit(int d, int u)
    {
        return (u ^ ((((d >> 1) & 7) ^ ((d >> 4) & 3)) & (TS / 8 - 1))) * 16;
    }
};

// What a thread stages of TS tokens (by roles, half of the waves the keys and half
// the values, a prompt of 8192 took 1.25 ms, 1.20 so): N items of EK elements of a key, and N items
// of DV elements of four tokens' values.  Every thread has some of both, so that
// no step carries a branch, and the items come to pieces of a pair of values each,
// which the main loop spreads between its matrix products.  The items of a wave
// lie in one 16-token group, which is one page's: where it is read from is the
// same for all lanes, and is kept and worked out in scalar registers.
template <int D, int TS, int NT>
struct Share {
    static constexpr int ALL = TS * D / NT;  // elements of a thread
    static constexpr int EK = std::min({ALL, D / 4, 32}), DV = std::min({ALL / 4, D / 16, 8});
    static constexpr int N = ALL / EK;
    static constexpr int PAIRS = N * EK / 2;  // and of the values, N * DV * 2 as many
    static_assert(N * DV * 4 == ALL && N * EK == ALL, "items cover the tokens");
    static constexpr int KL = D / EK, VL = D / DV;  // items of a token, of four tokens
    static_assert(KL >= 4 && VL >= 16, "a wave's items lie in one 16-token group");
};

template <int D, int TS, int NT, bool ONE>
struct Ahead {
    using S = Share<D, TS, NT>;
    using St = Stage<D, TS>;
    const PagedAttnArgs &a;
    const Work &w;
    int h, wave, lane;
    int pmin, after;                 // every row sees the tokens behind after, up to pmin
    int *spoiled;                    // this wave's, in LDS
    int64_t krow[S::N], vrow[S::N];  // pool rows of the groups of the next read, or -1
    int vt[S::N];                    // first token of the values' group
    uint32_t kc[S::N][S::EK / 8];    // codes
    uint32_t vc[S::N][4];
    uint32_t ks[S::N], kz[S::N];     // constants: a key's, and those of four tokens
    uint2 vs[S::N], vz[S::N];
    int kok[S::N];                   // the page of the key that was read exists

    // A key item: token ktok of the stage, element ke on.
    __device__ int kitem(int i) const
    {
        return i * NT + wave * 64 + lane;
    }
    __device__ int ktok(int i) const
    {
        return kitem(i) / S::KL;
    }
    // Element of its dword wd of codes: neighbouring lanes' units side by side
    // where a row is one group.
    __device__ int ke(int i, int wd) const
    {
        const int s = kitem(i) % S::KL;
        return ONE ? (s + wd * S::KL) * 8 : s * S::EK + wd * 8;
    }
    // A values item: quad vq of the tokens of group vgroup, dimension vd on.  A
    // wave has 16 runs of dimensions of four quads, dealt to the lanes so that 16
    // of them write to all banks.
    __device__ int vblock(int i) const
    {
        return i * (NT / 64) + wave;
    }
    __device__ int vgroup(int i) const
    {
        return vblock(i) / (S::VL / 16);
    }
    __device__ int vq() const
    {
        return (lane >> 5) | (lane >> 2 & 2);
    }
    __device__ int vd(int i) const
    {
        return (vblock(i) % (S::VL / 16) * 16 + ((lane & 7) | (lane >> 1 & 8))) * S::DV;
    }

    __device__ __forceinline__ int64_t group_row(int t) const
    {
        t = __builtin_amdgcn_readfirstlane(t);
        const int64_t row = pool_row(a.map, a.hkv, w.b, t);
        return row >= 0 ? row + (int64_t)h * a.map.page : -1;
    }
    __device__ __forceinline__ void look_keys(int t0)
    {
#pragma unroll
        for (int i = 0; i < S::N; ++i)
            krow[i] = group_row(t0 + ((i * NT + wave * 64) / S::KL & ~15));
    }
    __device__ __forceinline__ void look_values(int t0)
    {
#pragma unroll
        for (int i = 0; i < S::N; ++i) {
            vt[i] = t0 + vgroup(i) * 16;
            vrow[i] = group_row(vt[i]);
        }
    }

    // Groups of no page are read at row 0 of the pool (a pool has whole pages, of
    // 16 rows at least) and take no part: a key by `kok`, values by constants of 0.
    __device__ __forceinline__ void read_keys()
    {
        const int ng = ONE ? 1 : D / a.G;
#pragma unroll
        for (int i = 0; i < S::N; ++i) {
            kok[i] = krow[i] >= 0;
            const int64_t row = kok[i] ? krow[i] : 0;
            const uint32_t t = ktok(i) & 15, g = t * ng + (ONE ? 0 : ke(i, 0) / a.G);
#pragma unroll
            for (int wd = 0; wd < S::EK / 8; ++wd)
                kc[i][wd] = *reinterpret_cast<const uint32_t *>(
                    a.kp.c + row * (D / 2) + (t * (D / 2) + ke(i, wd) / 2));
            ks[i] = (a.kp.s + row * ng)[g];
            kz[i] = (a.kp.z + row * ng)[g];
        }
    }
    __device__ __forceinline__ void read_values()
    {
        const int ng = ONE ? 1 : D / a.G;
#pragma unroll
        for (int i = 0; i < S::N; ++i) {
            const bool in = vrow[i] >= 0;
            const int64_t row = in ? vrow[i] : 0;
            const uint32_t t = 4 * vq();
            const uint8_t *src = a.vp.c + row * (D / 2) + (t * (D / 2) + vd(i) / 2);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if constexpr (S::DV == 8)
                    vc[i][x] = *reinterpret_cast<const uint32_t *>(src + x * (D / 2));
                else if constexpr (S::DV == 4)
                    vc[i][x] = *reinterpret_cast<const uint16_t *>(src + x * (D / 2));
                else
                    vc[i][x] = src[x * (D / 2)];
            }
            if constexpr (ONE) {  // four tokens' constants lie side by side
                vs[i] = *reinterpret_cast<const uint2 *>(a.vp.s + row + t);
                vz[i] = *reinterpret_cast<const uint2 *>(a.vp.z + row + t);
            } else {
                uint32_t s[4], z[4];
                const uint32_t g = t * ng + vd(i) / a.G;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    s[x] = (a.vp.s + row * ng)[g + x * ng];
                    z[x] = (a.vp.z + row * ng)[g + x * ng];
                }
                vs[i] = make_uint2(s[0] | (s[1] << 16), s[2] | (s[3] << 16));
                vz[i] = make_uint2(z[0] | (z[1] << 16), z[2] | (z[3] << 16));
            }
            // Tokens that a row does not see take a weight of 0 in it, and 0 times what
            // is not finite would be NaN: those that no row sees (slots that were never
            // written) are taken as 0, and so are those of the others that are not
            // finite, which the rows that see them take at the end (add_spoiled).
            const int g0 = __builtin_amdgcn_readfirstlane(vt[i]);
            if (__builtin_expect(!(in & (g0 + 15 <= pmin) & (g0 > after)), 0)) {
                uint32_t keep[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int tt = g0 + (int)t + x;
                    keep[x] = (in & (tt < w.hi) & ((tt >= w.low) | (tt < a.sinks))) ? 0xFFFFu : 0u;
                }
                const uint32_t k01 = keep[0] | (keep[1] << 16), k23 = keep[2] | (keep[3] << 16);
                vs[i] = make_uint2(vs[i].x & k01, vs[i].y & k23);
                vz[i] = make_uint2(vz[i].x & k01, vz[i].y & k23);
                const uint32_t b01 = spoils(vs[i].x, vz[i].x), b23 = spoils(vs[i].y, vz[i].y);
                if (b01 | b23) {
                    const uint32_t m01 = ~((b01 >> 15) * 0xFFFFu), m23 = ~((b23 >> 15) * 0xFFFFu);
                    vs[i] = make_uint2(vs[i].x & m01, vs[i].y & m23);
                    vz[i] = make_uint2(vz[i].x & m01, vz[i].y & m23);
                    *spoiled = 1;
                }
            }
        }
    }

    // Pair x of the keys (pairs in nib_order): a 16-byte unit is written with its
    // fourth.
    uint32_t unit[4];
    __device__ __forceinline__ void put_keys(St &st, int x, const NibConst &nk)
    {
        const int i = x / (S::EK / 2), y = x % (S::EK / 2), wd = y / 4, j = y & 3;
        const h2v s = bits_h2(perm_b32(ks[i], ks[i], 0x01000100u));
        const h2v z = bits_h2(perm_b32(kz[i], kz[i], 0x01000100u));
        const uint32_t c = j & 2 ? kc[i][wd] >> 8 : kc[i][wd];
        const h2v v = fma2(j & 1 ? nib_pair<true>(c, nk) : nib_pair<false>(c, nk), s, z);
        unit[j] = __builtin_bit_cast(uint32_t, v);
        if (j == 3) {
            *reinterpret_cast<uint4 *>(st.k + (ktok(i) * St::KP + ke(i, wd) * 2)) =
                make_uint4(unit[0], unit[1], unit[2], unit[3]);
            if (wd == 0)
                st.ok[ktok(i) >> 4] = kok[i];  // (the lanes of a group write the same)
        }
    }
    // Pair x of the values: dimension x / 2, tokens 0, 1 or 2, 3; a dimension's
    // four tokens are written with its second.
    uint32_t vpair;
    __device__ __forceinline__ void put_values(St &st, int x, const NibConst &nk)
    {
        const int i = x / (S::DV * 2), y = x % (S::DV * 2), e = y >> 1;
        const uint32_t bt = e >> 1;
        // byte bt of two tokens in bytes 0 and 2
        const uint32_t sel = bt | 0x0C00u | ((4 + bt) << 16) | 0x0C000000u;
        const uint32_t c = y & 1 ? perm_b32(vc[i][3], vc[i][2], sel) : perm_b32(vc[i][1], vc[i][0], sel);
        const h2v s = bits_h2(y & 1 ? vs[i].y : vs[i].x), z = bits_h2(y & 1 ? vz[i].y : vz[i].x);
        const uint32_t v = __builtin_bit_cast(
            uint32_t, fma2(e & 1 ? nib_pair<true>(c, nk) : nib_pair<false>(c, nk), s, z));
        if (!(y & 1)) {
            vpair = v;
        } else {
            // quad q of a group: lane half q % 2, second 8 bytes for q / 2
            const int q = vq(), d = vd(i) + e;
            *reinterpret_cast<uint2 *>(st.v + (St::vrow(d) + St::vunit(d, 2 * vgroup(i) + (q & 1)) +
                                               (q >> 1) * 8)) = make_uint2(vpair, v);
        }
    }
};

// Block id -> (slot, split, cache head): heads next to each other, so that with
// eight of them each XCD keeps to one head's cache.  Which split comes first moves
// on with the slot: blocks are dealt to the parts of an XCD in turn, and the last
// splits of a short sequence have nothing to do (64 sequences of 1 .. 8192 tokens
// took 87 us with the splits in order, 77 so).
struct Place {
    int slot, split, h;
};

__device__ __forceinline__ Place place(const PagedAttnArgs &a)
{
    const uint32_t id = blockIdx.x;
    const uint32_t rest = id / (uint32_t)a.hkv;
    Place p;
    p.h = (int)(id % (uint32_t)a.hkv);
    const uint32_t s = rest / (uint32_t)a.splits;
    p.split = (int)((rest + s) % (uint32_t)a.splits);
    p.slot = (int)s;
    return p;
}

// The arguments (a kernel's first) once more, for code that hardly ever runs: their
// fields would otherwise be kept for it in scalar registers through the main loop.
__device__ __forceinline__ PagedAttnArgs args_again()
{
    auto p = (const __attribute__((address_space(4))) PagedAttnArgs *)(
        __builtin_amdgcn_kernarg_segment_ptr());
    asm volatile("" : "+s"(p));
    return *(const PagedAttnArgs *)p;
}

// One row of a block by one wave, token by token, a token seen or not touched at
// all: for blocks of few rows in several groups that hold a value that is not finite
// and that only some of the rows see, since the products of all rows with all tokens
// would make 0 times it of the others.  (64 sequences of 4 new tokens: 80 us, 2.6 ms
// so.)  64 scores at a time, a token a lane; then each seen token's value, D /
// 64 elements a lane.  The result goes where the block's goes.
template <int D>
__device__ __forceinline__ void row_alone(const PagedAttnArgs &a, const Work &w, const Place &pl, int row)
{
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63, ng = D / a.G;
    const int qi = row / a.rep, p = w.pos0 + qi, head = pl.h * a.rep + (row - qi * a.rep);
    const int64_t trow = w.tok0 + qi;
    const uint16_t *q = a.q + trow * a.q_stride + (int64_t)head * D;
    const int first = a.window > 0 ? p - a.window : -1;
    const float inf = __builtin_inff(), c2 = a.sm_scale * 1.44269504088896340736f;
    float m = -inf, l = 0.0f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        o[e] = 0.0f;
    const int begin = pl.split * w.per, end = min(w.steps, begin + w.per);
#pragma unroll 1
    for (int i = begin; i < end; ++i) {
        const int t = paged::step_token(w, i) + lane;
        int64_t at = pool_row(a.map, a.hkv, w.b, t);
        const bool see = at >= 0 && t <= p && (t > first || t < a.sinks);
        const uint64_t seen = __ballot(see);
        if (seen == 0)
            continue;
        at = see ? at + (int64_t)pl.h * a.map.page : 0;
        float x = 0.0f;
#pragma unroll 4
        for (int k = 0; k < D / 8; ++k) {
            const uint32_t c = *reinterpret_cast<const uint32_t *>(a.kp.c + at * (D / 2) + 4 * k);
            const int64_t gi = at * ng + 8 * k / a.G;
            const float s = h2f(a.kp.s[gi]), z = h2f(a.kp.z[gi]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x = __builtin_fmaf(h2f(q[8 * k + e]),
                                   __builtin_fmaf((float)((c >> (4 * e)) & 15u), s, z), x);
        }
        x = see ? x * c2 : -inf;
        float mn = x;
        static_for<6>([&](auto J) { mn = lane_max<J>(mn); });
        mn = fmaxf(m, mn);
        const float ms = mn > -inf ? mn : 0.0f;
        const float f = m > -inf ? __builtin_amdgcn_exp2f(m - ms) : 0.0f;
        const float wt = see ? __builtin_amdgcn_exp2f(x - ms) : 0.0f;
        m = mn;
        l = l * f + wt;
#pragma unroll
        for (int e = 0; e < E; ++e)
            o[e] *= f;
#pragma unroll 1
        for (int j0 = 0; j0 < 64; j0 += 8)
#pragma unroll
            for (int j = j0; j < j0 + 8; ++j) {
                const int64_t aj = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), j) << 32) |
                                             (uint32_t)__builtin_amdgcn_readlane((int)at, j));
                const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), j));
                const uint8_t *c = a.vp.c + aj * (D / 2) + lane * E / 2;
                const int64_t gi = aj * ng + lane * E / a.G;
                const float s = h2f(a.vp.s[gi]), z = h2f(a.vp.z[gi]);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int sh = E == 1 ? (lane & 1) * 4 : (e & 1) * 4;
                    const float v = __builtin_fmaf((float)((c[e / 2] >> sh) & 15), s, z);
                    o[e] = __builtin_fmaf(wj, seen >> j & 1 ? v : 0.0f, o[e]);
                }
            }
    }
    for (int d = 1; d < 64; d <<= 1)
        l += __shfl_xor(l, d);
    if (w.used == 1) {
        const float f = l > 0.0f ? 1.0f / l : 0.0f;
        uint16_t *dst = a.out + trow * a.out_stride + (int64_t)head * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
            dst[e] = f2h(o[e] * f);
    } else {
        const int64_t pr = part_of(a, w, row, pl.h) + pl.split;
#pragma unroll
        for (int e = 0; e < E; ++e)
            a.part_o[pr * D + lane * E + e] = o[e];
        if (lane == 0)
            *reinterpret_cast<float2 *>(a.part_ml + 2 * pr) = make_float2(m, l);
    }
}

// What a row of a tile takes from the values of group g0 that are not finite, this
// lane's half of its dimensions.  m is its final reference; its sum has these tokens'
// weights already.  (A prompt of 8192 takes 1.2 ms, with such a value in its last
// token as much, with nothing else in its cache 2.4 ms.  The look at each group that
// some rows see and some do not costs short prompts and windows 1 to 2%.)
template <int D>
__device__ __forceinline__ void add_spoiled(const PagedAttnArgs &a, const Work &w, int h, int g0, int p,
                                            const uint16_t *q, float m, v16f *o)
{
    const int lane = threadIdx.x & 63, hf = lane >> 5, ng = D / a.G;
    int64_t row = pool_row(a.map, a.hkv, w.b, g0);
    if (row < 0)
        return;
    row += (int64_t)h * a.map.page;
    bool odd = false;
    const int tl = g0 + (lane & 15);
    if (tl < w.hi && (tl >= w.low || tl < a.sinks))
        for (int x = 0; x < ng; ++x) {
            const int64_t gi = (row + (lane & 15)) * ng + x;
            odd |= (spoils(a.vp.s[gi], a.vp.z[gi]) & 0x8000u) != 0;
        }
    const NibConst nk = nib_const();
    for (uint32_t left = (uint32_t)__ballot(odd) & 0xFFFFu; left; left &= left - 1) {
        const int t = g0 + __builtin_ctz(left);
        const int64_t r1 = row + (t - g0);
        float x = 0.0f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {  // as the matrix product has them
            const int e = 16 * k + 8 * hf;
            const v8h qv = __builtin_bit_cast(v8h, nib_order(*reinterpret_cast<const uint4 *>(q + e)));
            const uint32_t c = *reinterpret_cast<const uint32_t *>(a.kp.c + r1 * (D / 2) + e / 2);
            const uint32_t s1 = a.kp.s[r1 * ng + e / a.G], z1 = a.kp.z[r1 * ng + e / a.G];
            const h2v s = bits_h2(s1 | s1 << 16), z = bits_h2(z1 | z1 << 16);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint32_t cy = y & 2 ? c >> 8 : c;
                const h2v kv = fma2(y & 1 ? nib_pair<true>(cy, nk) : nib_pair<false>(cy, nk), s, z);
                x = __builtin_fmaf((float)kv[0], (float)qv[2 * y], x);
                x = __builtin_fmaf((float)kv[1], (float)qv[2 * y + 1], x);
            }
            __builtin_amdgcn_sched_barrier(0);  // (all loads at once take registers that D = 256 lacks)
        }
        const auto sw =
            __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = (__uint_as_float(sw[0]) + __uint_as_float(sw[1])) * (a.sm_scale * 1.44269504088896340736f);
        const bool see = t <= p && (a.window == 0 || t > p - a.window || t < a.sinks);
        const float wt = __builtin_amdgcn_exp2f(x - (m > -__builtin_inff() ? m : 0.0f));
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int e = 32 * d + 2 * r + 4 * hf;
                const uint32_t c = *reinterpret_cast<const uint16_t *>(a.vp.c + r1 * (D / 2) + e / 2);
                const uint16_t s1 = a.vp.s[r1 * ng + e / a.G], z1 = a.vp.z[r1 * ng + e / a.G];
                const bool take = see && (spoils(s1, z1) & 0x8000u) != 0;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float v = __builtin_fmaf((float)((c >> (4 * y)) & 15u), h2f(s1), h2f(z1));
                    o[d][r + y] = __builtin_fmaf(take ? wt : 0.0f, take ? v : 0.0f, o[d][r + y]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// 32 query rows for each of NW waves.
template <int D, int NW, bool ONE>
__global__ __launch_bounds__(64 * NW)
    __attribute__((amdgpu_waves_per_eu(NW == 8 ? 2 : 1, NW == 8 ? 2 : 1))) void k_paged_tile(PagedAttnArgs a, int slots)
{
    constexpr int NT = 64 * NW, MR = 32 * NW;
    constexpr int KS = D / 16, DB = D / 32;
    // A stage holds 64 tokens, 32 for D = 256 and for two waves, of which then two
    // blocks fit a CU (16 sequences of one row over 8192: 142 us so, 197 with 64).  While one's scores are taken and
    // the last one's values are added, the next but one is written.
    constexpr int TS = D == 256 || NW == 2 ? 32 : 64, NB = TS == 32 ? 4 : 3;
    using St = Stage<D, TS>;
    using Sh = Share<D, TS, NT>;
    __shared__ __align__(16) St st[NB];
    __shared__ int spoiled[NW];  // by wave: it left out values that are not finite
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 31, hf = lane >> 5;
    Place pl = place(a);
    pl.slot = slots - 1 - pl.slot;  // late ones, the long rows of a prompt, first
    const Work w = find_work<MR>(a, pl.slot);
    if (w.rows == 0 || pl.split >= w.used)
        return;
    const float inf = __builtin_inff();
    const float c2 = a.sm_scale * 1.44269504088896340736f;  // log2(e)

    // this lane's query (past the last row, the last one again)
    const int row = w.row0 + wave * 32 + n, qrow = min(row, w.rows - 1), qi = qrow / a.rep;
    const int p = w.pos0 + qi, head = pl.h * a.rep + (qrow - qi * a.rep);
    const int64_t trow = w.tok0 + qi;
    const uint16_t *qr = a.q + trow * a.q_stride + (int64_t)head * D;
    uint4 qraw[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k)
        qraw[k] = *reinterpret_cast<const uint4 *>(qr + 16 * k + 8 * hf);

    v16f o[DB];
    float m = -inf, l = 0.0f;  // reference (log2 units); this lane's half of the sum
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[d][r] = 0.0f;

    const int begin = pl.split * w.per, end = min(w.steps, begin + w.per);
    const int pmin = w.pos0 + w.row0 / a.rep, pmax = w.pos0 + (min(w.row0 + MR, w.rows) - 1) / a.rep;

    auto weight = [&](const v16f &s, v8h *pb, float ms, int r) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -ms));
        pb[r >> 3][r & 7] = (_Float16)e;
        return e;
    };
    // scores of tokens t0 .. t0 + 31 (register r holds t0 + 8 (r / 4) + 4 hf +
    // r % 4) that a query does not see
    auto hide = [&](v16f &s, int t0, const int *ok) {
        const int first = a.window > 0 ? p - a.window : -1;  // up to here only as sinks
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int t = t0 + 8 * (r >> 2) + 4 * hf + (r & 3);
            const bool see = (t <= p) & ((t > first) | (t < a.sinks)) & (ok[r >> 3] != 0);
            s[r] = see ? s[r] : -inf;
        }
    };
    // Takes the weights' sums; where they pass what fp16 holds, or there is no
    // reference yet, the reference moves to the largest score.
    auto settle = [&](const v16f &s, v8h *pb, float sum) {
        if (__builtin_expect(__any(!(sum <= 0x1p15f) | (m == -inf)), 0)) {
            float mt = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r)
                mt = fmaxf(mt, s[r]);
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt),
                                                             __float_as_uint(mt), false, false);
            const float mn =
                fmaxf(m, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2 - TOP_TILE);
            const float ms = mn > -inf ? mn : 0.0f;  // nothing seen so far: weights 0
            const float f = m > -inf ? __builtin_amdgcn_exp2f(m - ms) : 0.0f;
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    o[d][r] *= f;
            sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sum += weight(s, pb, ms, r);
        }
        l += sum;
    };
    // One round of 32 tokens: the softmax of the scores sc, while the matrix cores
    // take the next round's scores sn (half uk of stage sk) and add the last
    // round's values (half uv of stage sv, weights pp).  A wave issues in order,
    // so the two overlap only where they alternate: each of 2 KS parts has its
    // share of the products, of the softmax, of the reads of a part ahead, and of
    // the staging (also(c)), and the scheduler is kept from gathering them.
    auto round = [&](const v16f &sc, v16f &sn, const v8h *pp, v8h *pb, const St &sk, int uk,
                     const St &sv, int uv, const v8h *qb, auto also) {
        const uint8_t *kb = sk.k + (n * St::KP + hf * 16), *vr = sv.v + St::vrow(n);
        const uint8_t *vb[2] = {vr + St::vunit(n, 4 * uv + hf), vr + St::vunit(n, 4 * uv + 2 + hf)};
        auto kfrag = [&](int k) {
            return *reinterpret_cast<const v8h *>(kb + (32 * uk * St::KP + 32 * k));
        };
        auto vfrag = [&](int c) {
            const int db = c % DB;
            return *reinterpret_cast<const v8h *>(vb[(c / DB) ^ (db & 1)] + 32 * db * St::VP);
        };
        constexpr int AHEAD = 2;
        v8h kf[KS], vf[2 * DB];  // KS == 2 DB
        float ls[2] = {0.0f, 0.0f};
        const float ms = m > -inf ? m : 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            sn[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < AHEAD; ++c) {
            kf[c] = kfrag(c);
            vf[c] = vfrag(c);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < KS; ++c) {
            sn = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[c], qb[c], sn, 0, 0, 0);
            if (c + AHEAD < KS)
                kf[c + AHEAD] = kfrag(c + AHEAD);
#pragma unroll
            for (int r = 16 * c / KS; r < 16 * (c + 1) / KS; r += 2) {
                if (KS == 16 && (c & 1))
                    continue;  // a part's share is one weight: two with every other
                ls[0] += weight(sc, pb, ms, r);
                ls[1] += weight(sc, pb, ms, r + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            o[c % DB] =
                __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[c], pp[c / DB], o[c % DB], 0, 0, 0);
            if (c + AHEAD < KS)
                vf[c + AHEAD] = vfrag(c + AHEAD);
            also(c);
            __builtin_amdgcn_sched_barrier(0);
        }
        settle(sc, pb, ls[0] + ls[1]);
    };

    if (begin < end) {
        constexpr int H = 64 / TS;      // stages of a step
        constexpr int PM = Sh::PAIRS / KS;  // pairs with a part
        const NibConst nk = nib_const();
        // first token of stage j; past the last one, the last one again
        auto token0 = [&](int j) {
            const int k = min(j, (end - begin) * H - 1);
            return paged::step_token(w, begin + k / H) + k % H * TS;
        };
        spoiled[wave] = 0;
        Ahead<D, TS, NT, ONE> ah{a, w, pl.h, __builtin_amdgcn_readfirstlane(wave), lane,
                                 pmin, a.window > 0 ? pmax - a.window : -1, spoiled + wave};
        auto put_all = [&](auto &from, St &to) {
#pragma unroll
            for (int x = 0; x < Sh::PAIRS; ++x) {
                from.put_keys(to, x, nk);
                from.put_values(to, x, nk);
            }
        };
        auto next = [&](int j) {  // reads what was looked up, looks stage j up
            ah.read_keys();
            ah.look_keys(token0(j));
            ah.read_values();
            ah.look_values(token0(j));
        };
        // two stages' pages are looked up, then read, at once
        auto first = ah;
        first.look_keys(token0(0));
        first.look_values(token0(0));
        ah.look_keys(token0(1));
        ah.look_values(token0(1));
        first.read_keys();
        first.read_values();
        next(2);
        put_all(first, st[0]);
        if constexpr (TS == 32) {
            put_all(ah, st[1]);
            next(3);
        } else {  // the values follow in the first round
#pragma unroll
            for (int x = 0; x < Sh::PAIRS; ++x)
                ah.put_keys(st[1], x, nk);
            ah.read_keys();
            ah.look_keys(token0(3));
        }
        v8h qb[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k)
            qb[k] = __builtin_bit_cast(v8h, nib_order(qraw[k]));
        __syncthreads();

        v16f sa, sb;  // scores of this round and the next, in turn
        v8h pa[2], pb[2];  // weights likewise
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                pb[x][e] = (_Float16)0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            sa[r] = 0.0f;
#pragma unroll
        for (int k = 0; k < KS; ++k)
            sa = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                *reinterpret_cast<const v8h *>(st[0].k + n * St::KP + hf * 16 + 32 * k), qb[k], sa,
                0, 0, 0);
        const int stages = (end - begin) * H;
        if constexpr (TS == 64) {
            int last = 0, cur = 0;
            for (int j = 0; j < stages; ++j) {
                const int t0 = token0(j);
                const int nx = cur + 1 < NB ? cur + 1 : 0, n2 = nx + 1 < NB ? nx + 1 : 0;
                const int ok[4] = {st[cur].ok[0], st[cur].ok[1], st[cur].ok[2], st[cur].ok[3]};
                const bool edge = !(ok[0] & ok[1] & ok[2] & ok[3]) || t0 + TS - 1 > pmin ||
                                  (a.window > 0 && t0 <= pmax - a.window);
                if (edge)
                    hide(sa, t0, ok);
                round(sa, sb, pb, pa, st[cur], 1, st[last], 1, qb, [&](int c) {
#pragma unroll
                    for (int x = 0; x < PM; ++x)
                        ah.put_values(st[nx], c * PM + x, nk);
                });
                ah.read_values();
                ah.look_values(token0(j + 3));
                if (edge)
                    hide(sb, t0 + 32, ok + 2);
                __syncthreads();  // stage nx is whole, every wave is through with the last
                round(sb, sa, pa, pb, st[nx], 0, st[cur], 0, qb, [&](int c) {
#pragma unroll
                    for (int x = 0; x < PM; ++x)
                        ah.put_keys(st[n2], c * PM + x, nk);
                });
                ah.read_keys();
                ah.look_keys(token0(j + 4));
                last = cur;
                cur = nx;
            }
#pragma unroll
            for (int c = 0; c < KS; ++c)
                o[c % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                    *reinterpret_cast<const v8h *>(
                        st[last].v + St::vrow(32 * (c % DB) + n) +
                        St::vunit(32 * (c % DB) + n, 4 + c / DB * 2 + hf)),
                    pb[c / DB], o[c % DB], 0, 0, 0);
        } else {
            int last = 0, cur = 0;
            for (int j = 0; j < stages; j += 2)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int t0 = token0(j + h);
                    const int nx = (cur + 1) & 3, n2 = (cur + 2) & 3;
                    const int ok[2] = {st[cur].ok[0], st[cur].ok[1]};
                    const bool edge = !(ok[0] & ok[1]) || t0 + TS - 1 > pmin ||
                                      (a.window > 0 && t0 <= pmax - a.window);
                    if (edge)
                        hide(h ? sb : sa, t0, ok);
                    auto put = [&](int c) {
#pragma unroll
                        for (int x = 0; x < PM; ++x) {
                            ah.put_keys(st[n2], c * PM + x, nk);
                            ah.put_values(st[n2], c * PM + x, nk);
                        }
                    };
                    if (h)
                        round(sb, sa, pa, pb, st[nx], 0, st[last], 0, qb, put);
                    else
                        round(sa, sb, pb, pa, st[nx], 0, st[last], 0, qb, put);
                    next(j + h + 4);
                    __syncthreads();
                    last = cur;
                    cur = nx;
                }
#pragma unroll
            for (int c = 0; c < KS; ++c)
                o[c % DB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
                    *reinterpret_cast<const v8h *>(
                        st[last].v + St::vrow(32 * (c % DB) + n) +
                        St::vunit(32 * (c % DB) + n, c / DB * 2 + hf)),
                    pb[c / DB], o[c % DB], 0, 0, 0);
        }
        // values that read_values left out (the last stage's were read before the last
        // barrier)
        int any = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i)
            any |= spoiled[i];
        if (__builtin_expect(any != 0, 0)) {
            const PagedAttnArgs again = args_again();
            for (int i = begin; i < end; ++i)
                for (int g0 = paged::step_token(w, i), g1 = g0 + 64; g0 < g1; g0 += 16)
                    if (!(g0 + 15 <= ah.pmin && g0 > ah.after))
                        add_spoiled<D>(again, w, pl.h, g0, p, qr, m, o);
        }
    }

    const auto sw =
        __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float lt = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (row >= w.rows)
        return;
    if (w.used == 1) {
        const float f = lt > 0.0f ? 1.0f / lt : 0.0f;
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
        const int64_t pr = part_of(a, w, row, pl.h) + pl.split;
        float *dst = a.part_o + pr * D;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<float4 *>(dst + 32 * d + 2 * r + 4 * hf) =
                    make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
        if (hf == 0)
            *reinterpret_cast<float2 *>(a.part_ml + 2 * pr) = make_float2(m, lt);
    }
}

// ---- few query rows: single tokens, and a few that were guessed ahead -------
//
// k_paged_rows: up to 16 query rows (new tokens times the heads of a cache head)
// of a sequence, NG groups per cached row.  Four waves take the block's token
// blocks of 64 in turn, straight from memory to registers, 16 tokens at a time
// as in the dense decode kernels: A = the K codes as fp16 integers against B =
// the queries, then A = the weights against B = the V codes.  Where a row is one
// group, codes enter as they are, so that nothing of a key or value is rounded:
//   q . khat_t = ks_t (q . code_t) + kz_t sum(q),
//   sum_t p_t vhat_t = sum_t (p_t vs_t) code_t + sum_t p_t vz_t.
// A code c is or-ed into an fp16 significand: as 64 + c in the K operand, whose
// offset 64 sum(q) is taken off by the scores' initial accumulator (6 of
// binary32's 24 bits of scores that are far below it anyway), and as 1024 + c or
// 64 + c in the V operand, taken off by a packed add: an output over many tokens
// is small beside the sum of its weights, and offsets of 128 left in the
// products cost half an fp16 step over 32768 tokens.
//
// The weights p_t vs_t are two fp16 parts, an A operand each: the first truncated,
// the second what that leaves, to nearest (truncated as well, the products would be
// low and the zeros' sum would not, an offset of all outputs).  Together they are off
// by 2^-21 of the weight, or by 2^-25 where that is more.  So the reference m that is
// taken off the scores x (log2 units) follows the weights and not the scores: it makes
// the first step's largest weight 2^8 whatever the values' scale is, so that 2^-25 is
// 2^-33 of it, and moves when a weight passes 2^15.  (At 2^12 it moves so often that
// one sequence of 32768 takes 19.9 us instead of 18.8; at 1, 6000 tokens that together
// have 1% of the weight beside one of value 0 lost all of it to truncation.  Scales
// below 2^-24, none but 0 in fp16, count as that, so that rows of equal values have a
// reference.)
//
// Where a row is several groups, a key's constants belong to its elements and not to
// its score: keys and values enter as RN16(code * scale + zero), the weights
// rounded to fp16, as in the tiles, and m makes the largest score's weight 2^8.  (16 sequences
// over up to 8192 tokens, 32 heads on 8: 35 us with groups of 128, 38 of 64, 39 of
// 32; by 64-row tiles 142.)
//
// What bounds it: a stage of 32 tokens is 4.3 KB for D = 128 and about 280 vector
// instructions, 1100 cycles of a SIMD where the memory's share of one takes 2000;
// but of the 17 us that a block of 1024 tokens takes 7 are its start (sequence,
// pages, queries, first codes) and its end, which four blocks a CU hide only in
// part.  64 sequences of 1 .. 8192 tokens: 70 us and 6 for their joining, 277 MB.
// A wave's codes and constants come through a ring of its own in LDS, 32 tokens
// a stage, by loads that go from memory straight there (16 bytes a lane): the
// next stage is on its way while this one is multiplied, at no registers, and
// the lanes take each cached row in the pieces that the matrix operands want.
constexpr int ROWS_W = 4;   // waves of a block
constexpr int ROWS_NS = 2;  // stages of a wave's ring

template <int D, int NG>
struct RowsRing {
    static constexpr int KB = 32 * D / 2;  // bytes of a stage's K codes, and of its V codes
    static constexpr int STAGE = 2 * KB + 256 * NG;  // and ks, kz, vs, vz of 32 tokens
    static constexpr int LOADS = 2 * (KB / 1024) + NG;
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

template <int D, int NG>
__global__ __launch_bounds__(64 * ROWS_W)
    __attribute__((amdgpu_waves_per_eu(D == 256 ? 2 : 4, D == 256 ? 2 : 4))) void k_paged_rows(PagedAttnArgs a)
{
    using Ring = RowsRing<D, NG>;
    constexpr int G = D / NG;
    constexpr int MR = paged::FEW_ROWS;
    constexpr int KW = D / 32;  // dwords of K codes of a lane: D / 4 elements of a token
    constexpr int VD = D / 16;  // dimensions of a lane in the value product
    constexpr int RED = ROWS_W * MR * (D + 2) * 4, RING = ROWS_W * ROWS_NS * Ring::STAGE;
    __shared__ __align__(16) uint8_t lds[RED > RING ? RED : RING];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 15, g = lane >> 4;
    const Place pl = place(a);
    const float inf = __builtin_inff();
    const float c2 = a.sm_scale * 1.44269504088896340736f;  // log2(e)
    const Work w = few_work(a, pl.slot);
    if (w.rows == 0 || pl.split >= w.used)
        return;
    const int R = min(MR, w.rows - w.row0);

    // this lane's query (column n of the scores)
    const int row = w.row0 + min(n, R - 1), qi = row / a.rep;
    const int p = w.pos0 + qi;
    const int wfirst = a.window > 0 ? p - a.window : -1;
    const int pmin = w.pos0 + w.row0 / a.rep, pmax = w.pos0 + (w.row0 + R - 1) / a.rep;
    uint4 qraw[KW];
    {
        const uint16_t *qr = a.q + (int64_t)(w.tok0 + qi) * a.q_stride +
                             (int64_t)(pl.h * a.rep + (row - qi * a.rep)) * D + (D / 4) * g;
#pragma unroll
        for (int k = 0; k < KW; ++k)
            qraw[k] = *reinterpret_cast<const uint4 *>(qr + 8 * k);
    }
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
    // constants: [array][16-token group][token][group of the row], 256 bytes a load
    const uint16_t *carr[NG];
    int cgrp[NG];
#pragma unroll
    for (int x = 0; x < NG; ++x) {
        const int b = 256 * x + 4 * lane, arr = b / (64 * NG), rem = b % (64 * NG);
        cgrp[x] = rem / (32 * NG);
        carr[x] = (arr < 2 ? arr ? a.kp.z : a.kp.s : arr < 3 ? a.vp.s : a.vp.z) + rem % (32 * NG) / 2;
    }

    int64_t base = -1;  // pool rows of the next 64 groups of 16 tokens, one a lane
    auto look = [&](int k) {
        const int kk = k + (lane >> 1);
        base = -1;
        if (kk < stages) {
            const int t = token_at(kk) + 16 * (lane & 1);
            if (t < w.hi)
                base = pool_row(a.map, a.hkv, w.b, t);
            if (base >= 0)
                base += (int64_t)pl.h * a.map.page;
        }
    };
    auto issue = [&](int k) -> int {
        if (k > 0 && (k & 31) == 0)
            look(k);
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
#pragma unroll
        for (int x = 0; x < NG; ++x)
            dma4(carr[x] + (cgrp[x] ? r0[1] : r0[0]) * NG, at + 2 * Ring::KB + 256 * x);
        return ok;
    };

    look(0);  // on its way together with the queries
    v8h qb[KW];
    float qsum = 0.0f;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
        qb[k] = __builtin_bit_cast(v8h, nib_order(qraw[k]));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            qsum += (float)qb[k][e];
    }
    {
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
        // one group a row: constants of tokens 4 g + r, + 64 array + 32 group
        const uint8_t *cst = stg + 2 * Ring::KB + 8 * g;
        auto constant = [&](int arr, int u, int token, int grp) {
            return (uint32_t)*reinterpret_cast<const uint16_t *>(
                stg + 2 * Ring::KB + (64 * NG * arr + 32 * NG * u) + (token * NG + grp) * 2);
        };
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
            if constexpr (NG > 1) {
                // this lane's piece of token n lies in one group, or in two halves in two
                constexpr int PG = NG > 4 ? NG / 4 : 1;
                v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < PG; ++p) {
                    const int grp = (D / 4 * g + 8 * (p * (KW / PG))) / G;
                    const uint32_t ks = constant(0, u, n, grp), kz = constant(1, u, n, grp);
                    const h2v s = bits_h2(ks | ks << 16), z = bits_h2(kz | kz << 16);
#pragma unroll
                    for (int c = p * (KW / PG); c < (p + 1) * (KW / PG); ++c) {
                        auto two = [&](uint32_t w, bool hi) {
                            return __builtin_bit_cast(
                                uint32_t, fma2(hi ? nib_pair<true>(w, nk) : nib_pair<false>(w, nk), s, z));
                        };
                        const uint4 kf = make_uint4(two(kc[c], false), two(kc[c], true),
                                                    two(kc[c] >> 8, false), two(kc[c] >> 8, true));
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, kf), qb[c],
                                                                     acc, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    x[u][r] = __builtin_fmaf(acc[r], c2, -ms);
                continue;
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
        const bool edge = ok != 3 || th + 31 > pmin || (a.window > 0 && th <= pmax - a.window);
        if (edge) {
            asm volatile("");  // a branch, not selects in every step
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int t = th + 16 * u + 4 * g + r;
                    const bool see = (ok >> u & 1) && t <= p && (t > wfirst || t < a.sinks);
                    x[u][r] = see ? x[u][r] : -inf;
                    if constexpr (NG > 1)
                        continue;
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
                    if constexpr (NG == 1)
                        zn = __builtin_fmaf(e, (float)vzh[u][r], zn);
                    wt[u][r] = NG == 1 ? __builtin_fmaf(e, (float)vsh[u][r], 0.0f) : e;
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
                    y = fmaxf(y, NG > 1 ? x[u][r]
                                        : x[u][r] + __builtin_amdgcn_logf(
                                                        fmaxf((float)vsh[u][r], 0x1p-24f)));
            y = lane_max<4>(y);
            y = lane_max<5>(y) - TOP_ROWS;
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
                if constexpr (NG > 1) {
                    const h2v w2 = {(_Float16)wt[u][r], (_Float16)wt[u][r + 1]};
                    hh[2 * u + r / 2] = __builtin_bit_cast(uint32_t, w2);
                    continue;
                }
                const h2v hi = pk_rtz(wt[u][r], wt[u][r + 1]);
                const h2v lo = {(_Float16)__builtin_fmaf((float)hi[0], -1.0f, wt[u][r]),
                                (_Float16)__builtin_fmaf((float)hi[1], -1.0f, wt[u][r + 1])};
                hh[2 * u + r / 2] = __builtin_bit_cast(uint32_t, hi);
                ll[2 * u + r / 2] = __builtin_bit_cast(uint32_t, lo);
            }
        const v8h wh = __builtin_bit_cast(v8h, make_uint4(hh[0], hh[1], hh[2], hh[3]));
        const v8h wl = NG > 1 ? v8h{} : __builtin_bit_cast(v8h, make_uint4(ll[0], ll[1], ll[2], ll[3]));
        // constants of the values' pairs of tokens, in this lane's dimensions' group
        h2v vs2[4], vz2[4];
        if constexpr (NG > 1) {
            const int grp = VD * n / G;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int u = x >> 1, t = 4 * g + 2 * (x & 1);
                uint32_t keep = 0xFFFFFFFFu;
                if (edge) {  // tokens that no row sees
                    auto held = [&](int tt) {
                        return (ok >> u & 1) && tt < w.hi && (tt >= w.low || tt < a.sinks);
                    };
                    keep = (held(th + 16 * u + t) ? 0xFFFFu : 0u) |
                           (held(th + 16 * u + t + 1) ? 0xFFFF0000u : 0u);
                }
                vs2[x] = bits_h2((constant(2, u, t, grp) | constant(2, u, t + 1, grp) << 16) & keep);
                vz2[x] = bits_h2((constant(3, u, t, grp) | constant(3, u, t + 1, grp) << 16) & keep);
            }
        }
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
                    if constexpr (NG > 1) {
                        lo[2 * u + t] = fma2(lo[2 * u + t], vs2[2 * u + t], vz2[2 * u + t]);
                        hi[2 * u + t] = fma2(hi[2 * u + t], vs2[2 * u + t], vz2[2 * u + t]);
                    }
                }
            const v8h vlo = {lo[0][0], lo[0][1], lo[1][0], lo[1][1],
                             lo[2][0], lo[2][1], lo[3][0], lo[3][1]};
            const v8h vhi = {hi[0][0], hi[0][1], hi[1][0], hi[1][1],
                             hi[2][0], hi[2][1], hi[3][0], hi[3][1]};
            o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, vlo, o[2 * bt], 0, 0, 0);
            if constexpr (NG == 1)
                o[2 * bt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl, vlo, o[2 * bt], 0, 0, 0);
            o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wh, vhi, o[2 * bt + 1], 0, 0, 0);
            if constexpr (NG == 1)
                o[2 * bt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(wl, vhi, o[2 * bt + 1], 0, 0, 0);
        }
    }

    if constexpr (NG > 1) {
        // Values that only some rows see have to be finite (weights of one group's rows
        // are masked row by row instead).  All waves look at all of them: no more than
        // 15 behind the first row's position, and as many where windows begin.  (Looked
        // at where they pass through, single tokens, which have none, took 41 us
        // instead of 39.)
        if (pmin != pmax) {
            const PagedAttnArgs again = args_again();
            const int behind = pmax - pmin, of = (again.window > 0 ? 2 : 1) * behind * NG;
            bool odd = false;
            for (int i = lane; i < of; i += 64) {
                const int j = i / NG;
                const int t = j < behind ? pmin + 1 + j : pmax - again.window - (j - behind);
                const int64_t at = pool_row(again.map, again.hkv, w.b, t);
                const int64_t gi = (at + (int64_t)pl.h * again.map.page) * NG + i % NG;
                if (at >= 0 && t < w.hi)
                    odd |= (spoils(again.vp.s[gi], again.vp.z[gi]) & 0x8000u) != 0;
            }
            if (__any(odd)) {
                for (int r = wave; r < R; r += ROWS_W)
                    row_alone<D>(again, w, pl, w.row0 + r);
                return;
            }
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
            const int64_t pr = part_of(a, w, rr, pl.h) + pl.split;
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
    __shared__ float red[WPR > 1 ? 4 : 1][D + 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int h = (int)(blockIdx.x % (uint32_t)a.hkv);
    const float inf = __builtin_inff();
    const int slot = (int)(blockIdx.x / (uint32_t)a.hkv);
    const Work w = MR == paged::FEW_ROWS ? few_work(a, slot) : find_work<MR>(a, slot);
    if (w.rows == 0 || w.used == 1)
        return;
    for (int r0 = blockIdx.y * RPB; r0 < MR && w.row0 + r0 < w.rows; r0 += gridDim.y * RPB) {
        const int r = r0 + wave / WPR, row = min(w.row0 + r, w.rows - 1), qi = row / a.rep;
        const bool live = r < MR && w.row0 + r < w.rows;
        const int head = h * a.rep + (row - qi * a.rep);
        const int64_t trow = w.tok0 + qi;
        const int64_t pr = part_of(a, w, row, h);
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
        // rows of a block row are shared by blocks of eight (16 in one block: 8
        // sequences of 4096 19 us instead of 18)
        hipLaunchKernelGGL((k_paged_combine<D, MR, 1>), dim3(x, MR == paged::FEW_ROWS ? 2 : MR / 32),
                           dim3(256), 0, s, a);
    return hipGetLastError();
}

template <int D, int NW>
hipError_t go_tile(const PagedAttnArgs &a, hipStream_t s)
{
    constexpr int MR = 32 * NW;
    const int slots = (int)paged::slots({a.which, MR}, a.map.T, a.map.B, a.rep);
    const dim3 grid((unsigned)((int64_t)slots * a.hkv * a.splits));
    if (a.G == D)
        hipLaunchKernelGGL((k_paged_tile<D, NW, true>), grid, dim3(64 * NW), 0, s, a, slots);
    else
        hipLaunchKernelGGL((k_paged_tile<D, NW, false>), grid, dim3(64 * NW), 0, s, a, slots);
    hipError_t e = hipGetLastError();
    return e != hipSuccess || a.splits == 1 ? e : go_combine<D, MR>(a, slots, s);
}

template <int D>
hipError_t go_few(const PagedAttnArgs &a, hipStream_t s)
{
    constexpr int MR = paged::FEW_ROWS;
    const int slots = (int)paged::slots({a.which, MR}, a.map.T, a.map.B, a.rep);
    const dim3 grid((unsigned)((int64_t)slots * a.hkv * a.splits));
    const dim3 block(64 * ROWS_W);
    switch (D / a.G) {
    case 1: hipLaunchKernelGGL((k_paged_rows<D, 1>), grid, block, 0, s, a); break;
    case 2: hipLaunchKernelGGL((k_paged_rows<D, 2>), grid, block, 0, s, a); break;
    case 4:
        if constexpr (D >= 128)
            hipLaunchKernelGGL((k_paged_rows<D, 4>), grid, block, 0, s, a);
        break;
    case 8:
        if constexpr (D >= 256)
            hipLaunchKernelGGL((k_paged_rows<D, 8>), grid, block, 0, s, a);
        break;
    }
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

hipError_t launch_paged_attention(const PagedAttnArgs &a, int rows, hipStream_t s)
{
    switch (a.D) {
    case 64: return go_rows<64>(a, rows, s);
    case 128: return go_rows<128>(a, rows, s);
    case 256: return go_rows<256>(a, rows, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace quarot
