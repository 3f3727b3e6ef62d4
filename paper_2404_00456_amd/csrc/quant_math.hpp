// The quantizers' arithmetic (division by a stored scale, rounding to codes)
// and 16-byte row accesses, shared by the rotate kernels and the paged append.
#pragma once

#include "common.hpp"

namespace quarot {

// The quantizers divide by a stored fp16 scale sf.  RN(y / sf) is formed
// with Markstein's correction from rf = RN(1 / sf), computed once per row or
// group: q0 = RN(y rf), e = y - q0 sf (exact, one fma), q = RN(q0 + e rf).
// With a correctly rounded reciprocal this equals the IEEE quotient except
// where it underflows (|q| < 2^-100), where both give code 0; checked
// against IEEE division for every positive fp16 divisor.  A zero or
// infinite scale gives code 0 (y / inf = 0 as well).
struct Divisor {
    float s, r;
    bool ok;
};

__device__ __forceinline__ Divisor make_divisor(float sf)
{
    Divisor d;
    d.s = sf;
    d.ok = sf > 0.0f && sf < __builtin_inff();
    d.r = d.ok ? 1.0f / sf : 0.0f;
    return d;
}

__device__ __forceinline__ float quotient(float y, const Divisor &d)
{
    const float q0 = y * d.r;
    const float e = __builtin_fmaf(-q0, d.s, y);
    return __builtin_fmaf(e, d.r, q0);
}

// RN(x / 15) without a division instruction: Markstein's correction from
// RN(1/15), exact for every binary32 x (checked exhaustively on the CPU).
__device__ __forceinline__ float div15(float x)
{
    const float r = 0x1.111112p-4f;  // RN32(1/15)
    const float q0 = x * r;
    return __builtin_fmaf(__builtin_fmaf(-q0, 15.0f, x), r, q0);
}

// Rounding to an integer code without conversion instructions: for t
// clamped to the code range (|t| < 2^22), t + 1.5 * 2^23 lies in
// [2^23, 2^24), where floats are spaced by 1, so the add rounds t to the
// nearest integer, ties to even, and the low bits of the sum's encoding are
// that integer in two's complement.  Clamping before rounding equals
// rounding before clamping, as the bounds are integers.
__device__ __forceinline__ uint32_t round_bits(float t)
{
    return __float_as_uint(t + 0x1.8p23f);
}

// Asymmetric uint4 code: clamp(rint_even(RN(RN(y - zf) / sf)), 0, 15), as
// the low nibble of the rounding sum's encoding (whose bits 4-21 are zero),
// for packing; the caller applies the zero-or-infinite-scale rule (code 0).
__device__ __forceinline__ uint32_t asym_code_bits(float y, const Divisor &d, float zf)
{
    return round_bits(fminf(fmaxf(quotient(y - zf, d), 0.0f), 15.0f));
}

__device__ __forceinline__ void unpack8(uint4 raw, float *v)
{
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = h2f((uint16_t)(w[i] & 0xFFFFu));
        v[2 * i + 1] = h2f((uint16_t)(w[i] >> 16));
    }
}

__device__ __forceinline__ void load8(const uint16_t *p, float *v)
{
    unpack8(*reinterpret_cast<const uint4 *>(p), v);
}

__device__ __forceinline__ void store8(uint16_t *p, const float *v)
{
    uint4 raw;
    raw.x = (uint32_t)f2h(v[0]) | ((uint32_t)f2h(v[1]) << 16);
    raw.y = (uint32_t)f2h(v[2]) | ((uint32_t)f2h(v[3]) << 16);
    raw.z = (uint32_t)f2h(v[4]) | ((uint32_t)f2h(v[5]) << 16);
    raw.w = (uint32_t)f2h(v[6]) | ((uint32_t)f2h(v[7]) << 16);
    *reinterpret_cast<uint4 *>(p) = raw;
}

}  // namespace quarot
