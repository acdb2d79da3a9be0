// Rows of activations in 8 bits.  Every 32 neighbours of a row (the last block of a row may be shorter) share a scale s: with a = max |x|
//     s = a / 127, rounded up to a bfloat16, at least 2^-126        q = the whole number nearest to x * (1 / s), ties to even
// in fp32, each step rounded once; what comes back is q s.  |q| <= 127 follows from s >= a / 127.  An element is off by at most s / 2 (and fp32's rounding of
// x * (1 / s)): by at most a / 252, (1/254) (1 + 2^-7) of its block's largest, where a >= 127 * 2^-126, and by 2^-127 in a block of smaller numbers, whose s is held at 2^-126.
// Rounded up in 8 bits of significand a scale takes 2 bytes of 32 elements, costs at most 2^-7 of the step
// and keeps q s exact in fp32 (7 bits times 8).  Whole numbers rather than 8-bit floats: their step is the same for all elements of a block, so the error of
// a sum of many of them is s / sqrt(12) an element, some 0.6 % of a normal block's standard deviation, where e4m3's 2^-4 half a step gives 2.6 %.
// A block with an infinity or a NaN has s = NaN and q = 0: all of it comes back as NaN.
#pragma once

#include "device_utils.h"

namespace {

constexpr int BLOCK8 = 32;
struct Scale8 { float s, inv; };                               // inv 0: not finite

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }   // as a whole number: a NaN is above infinity
// Both quotients are rounded as fp32 rounds: a product with the rounded 1 / 127, or a reciprocal to 1 ulp, and one correction by what it leaves over.  (The remainders are exact.  All 2^23
// significands of a, and the 128 of s with a reciprocal up to 2 ulp off, come to what a division gives; below 2^-126, where a quotient loses bits, s does not depend on it.
// A gated layer's tile takes no longer than without the corrections: 65536 rows, 1024 -> 2 x 2048, 728 us either way.)
__device__ __forceinline__ Scale8 scale8(uint32_t largest)
{
    if (largest >= 0x7f800000u) return Scale8{__uint_as_float(0x7fc00000u), 0.f};
    constexpr float R = 1.f / 127.f;
    const float a = __uint_as_float(largest), near = a * R, ratio = __builtin_fmaf(__builtin_fmaf(-127.f, near, a), R, near);
    const float s = __uint_as_float(max((__float_as_uint(ratio) + 0xffffu) & 0xffff0000u, 0x00800000u)), inv = __builtin_amdgcn_rcpf(s);
    return Scale8{s, __builtin_fmaf(__builtin_fmaf(-s, inv, 1.f), inv, inv)};
}
// of a lane's and that of the lane 32 further on or back
__device__ __forceinline__ uint32_t largest_of_halves(uint32_t v)
{
    const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);                // the lower half's twice, the upper half's twice
    return max(both[0], both[1]);
}
__device__ __forceinline__ bf16_t scale8_bits(const Scale8& s) { return bf16_t(__float_as_uint(s.s) >> 16); }
// four elements.  The product is rounded first, as the definition says; added to 1.5 * 2^23 it leaves its nearest whole number in the lowest bits of the sum.
__device__ __forceinline__ uint32_t pack8(float x0, float x1, float x2, float x3, float inv)
{
#pragma clang fp contract(off)
    constexpr float MAGIC = 12582912.f;
    auto low = [&](float x) { return __float_as_uint(x * inv + MAGIC); };
    const uint32_t q = __builtin_amdgcn_perm(__builtin_amdgcn_perm(low(x3), low(x2), 0x0c0c0400u), __builtin_amdgcn_perm(low(x1), low(x0), 0x0c0c0400u), 0x05040100u);
    return inv == 0.f ? 0u : q;
}
// element i of four
__device__ __forceinline__ float unpack8(uint32_t q, int i) { return float(int32_t(q << (24 - 8 * i)) >> 24); }

// up to 8 elements at any address; left: those that are there
__device__ __forceinline__ u32x2 load_eight(const int8_t* p, int left)
{
    typedef uint32_t u32x2_at1 __attribute__((ext_vector_type(2), aligned(1)));
    if (left >= 8) return *reinterpret_cast<const u32x2_at1*>(p);
    u32x2 v = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) v[i >> 2] |= uint32_t(uint8_t(p[i])) << (8 * (i & 3));
    return v;
}
__device__ __forceinline__ uint32_t load_four(const int8_t* p, int left)
{
    typedef uint32_t u32_at1 __attribute__((aligned(1)));
    if (left >= 4) return *reinterpret_cast<const u32_at1*>(p);
    uint32_t v = 0u;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) v |= uint32_t(uint8_t(p[i])) << (8 * i);
    return v;
}
__device__ __forceinline__ void store_eight(int8_t* p, int left, u32x2 v)
{
    typedef uint32_t u32x2_at1 __attribute__((ext_vector_type(2), aligned(1)));
    if (left >= 8) {
        *reinterpret_cast<u32x2_at1*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < left) p[i] = int8_t(v[i >> 2] >> (8 * (i & 3)));
}

}  // namespace
