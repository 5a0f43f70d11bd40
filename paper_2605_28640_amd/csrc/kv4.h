// Rows in 4 bits: 32 neighbouring channels share a power of two 2^e (one byte, e + 127; 255: the group is NaN), a channel is one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, the lower of two channels in the low half of a byte.  These are the operand types
// of the CDNA4 conversions: two channels of a row become a bfloat16 pair in one instruction, and exactly, since a value has two significant
// bits.  (The tests hold rows of every size of number, ties, both ends of the range, infinities and NaN against
// the definition, byte for byte; an infinite scale, which is what byte 255 gives, makes every value NaN.)
#pragma once

#include "common.h"

namespace rs {

constexpr int kKv4Group = 32;                  // channels that share a scale
constexpr int kKv4Least = 2, kKv4Most = 252;   // scale bytes that kv4_append writes: 2^-125 .. 2^125, so that no value is subnormal or infinite
constexpr uint32_t kKv4Nan = 255;

template <int D>
struct Kv4Row {
    static constexpr int CODES = D / 2, SCALES = D / kKv4Group;  // bytes a row
};

__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// byte SEL of a word of codes, times the scale
template <int SEL>
__device__ __forceinline__ uint32_t kv4_pair(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}
// the eight values of a word of codes as four bfloat16 pairs
__device__ __forceinline__ void kv4_values(uint32_t codes, float scale, uint32_t (&out)[4])
{
    out[0] = kv4_pair<0>(codes, scale);
    out[1] = kv4_pair<1>(codes, scale);
    out[2] = kv4_pair<2>(codes, scale);
    out[3] = kv4_pair<3>(codes, scale);
}

// The scale byte of a group whose largest magnitude has these bits: the smallest 2^e with at most 7 of them in it (7 is half
// way between 6 and the next value there would be, so nothing is further off than its rounding; larger e only near the end of the range).
__device__ __forceinline__ uint32_t kv4_scale_byte(uint32_t top)
{
    if (top >= 0x7f800000u) return kKv4Nan;
    const int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(e < kKv4Least ? kKv4Least : e > kKv4Most ? kKv4Most : e);
}
// eight values as codes, to nearest, ties to the even code
__device__ __forceinline__ uint32_t kv4_codes(const float (&x)[8], float scale)
{
    uint32_t c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
}

}  // namespace rs
