// Rows in 8 bits.  A row goes in groups of 64 elements, the last one filled up with zeros.  A group's scale is the smallest power of two 2^k with
// max |x| <= 127 * 2^k, at least 2^-126; its exponent byte is k + 127, that of a group with an infinity or NaN (or a number beyond fp32) 255, and such
// a group stands for NaN.  A code is rint(x / 2^k), ties to even.  The division is exact, so that the codes of given numbers are the same whatever
// computes them, and code * 2^k has 7 bits: it is exact in bf16.
#ifndef SPION_EIGHT_BIT_H_
#define SPION_EIGHT_BIT_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_common.h"
#include "spion_internal.h"

namespace spion {

constexpr int kGroup = 64;
constexpr int kNotFinite = 255;
constexpr float kMost = 3.4028234663852886e38f;   // fp32's largest number

// The exponent byte that a group whose largest magnitude is `most` has.  It grows with `most`: the largest byte of a group's parts is the group's.
// 127 * 2^-6 = 1 + 63 / 64: a mantissa beyond that takes the next power of two.
__device__ __forceinline__ int exponent_byte(float most) {
    const unsigned u = __builtin_bit_cast(unsigned, most);
    if (u >= 0x7f800000u) return kNotFinite;   // (`most` is not negative)
    const int e = (int)(u >> 23) - 6 + ((u & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return e < 1 ? 1 : e;
}
__device__ __forceinline__ int exponent_byte(double most) {
    if (!(most <= (double)kMost)) return kNotFinite;
    const unsigned long long u = __builtin_bit_cast(unsigned long long, most);
    const int e = (int)(u >> 52) - 1023 + 127 - 6 + ((u & 0xfffffffffffffull) > 0xfc00000000000ull ? 1 : 0);
    return e < 1 ? 1 : e;
}
// Whether a number off by up to 8 units of 2^-24 may have another exponent byte than `most`.
__device__ __forceinline__ bool near_border(float most) {
    return (__builtin_bit_cast(unsigned, most) & 0x7fffffu) - (0x7e0000u - 8u) <= 16u;
}
// The largest of eight lanes beside each other that have a group's 64 elements.
__device__ __forceinline__ int group_exponent(int e) {
    e = max(e, __shfl_xor(e, 1));
    e = max(e, __shfl_xor(e, 2));
    return max(e, __shfl_xor(e, 4));
}
__device__ __forceinline__ float eight_scale(int exponent) { return __builtin_bit_cast(float, (unsigned)exponent << 23); }   // 255: infinity, times code 0 NaN
// 2^-k, for 1 .. 249; of a group that is not finite 0, so that with finite numbers codes come out as 0
__device__ __forceinline__ float eight_inverse(int exponent) {
    return exponent == kNotFinite ? 0.f : __builtin_bit_cast(float, (unsigned)(254 - exponent) << 23);
}

typedef unsigned Codes8 __attribute__((ext_vector_type(2)));
template <typename S>
__device__ __forceinline__ Codes8 codes_of(const S (&v)[8], int exponent) {
    const S inv = (S)eight_inverse(exponent);
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = exponent == kNotFinite ? 0 : (int)__builtin_rint(v[i] * inv);
    Codes8 r;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        r[i] = (c[4 * i] & 0xff) | (c[4 * i + 1] & 0xff) << 8 | (c[4 * i + 2] & 0xff) << 16 | (unsigned)c[4 * i + 3] << 24;
    return r;
}
// The same for numbers off by up to 4 units of 2^-24; false if one of them may have another code.  127 * 4 * 2^-24 = 2^-15 less 1/128 of it.
__device__ __forceinline__ bool codes_of(Codes8& q, const float (&v)[8], int exponent) {
    constexpr float kRound = 12582912.f;   // 1.5 * 2^23: a sum with it has the nearest whole number (ties to even) in its low bits
    const float inv = eight_inverse(exponent);
    float far = 0.f;
    unsigned t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float sum = fmaf(v[i], inv, kRound);   // (a product with a power of two is exact)
        far = fmaxf(far, fabsf(fmaf(v[i], inv, -(sum - kRound))));
        t[i] = __builtin_bit_cast(unsigned, sum);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned lo = __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0c0c0400u), hi = __builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0c0c0400u);
        q[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
    return far < 0.5f - 0x1p-15f;
}
__device__ __forceinline__ void values_of(float (&v)[8], Codes8 codes, float scale) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(signed char)(codes[i / 4] >> (8 * (i % 4))) * scale;
}

}  // namespace spion
#endif
