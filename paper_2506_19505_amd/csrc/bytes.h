// Values of 8 bits, e4m3 (a sign, four bits of exponent, three behind the first one; 448 at most, NaN, no infinities), with a power of
// two as scale for kScaleRows rows of a head: what a cache in pages of 8 bits holds.
//
// Numbers.  s is the least of 2^-32 .. 2^8 with amax <= 448 s.  A value x is held as the nearest e4m3 to x / s, ties to even: off by at most
// 2^-4 of itself, or by 2^-10 s where it is below 2^-6 s.  Values beyond 61440, the largest number of four bits that fp16 has, count as
// that (off by 2^-4 at most as well).  Every value is then an fp16 number: x is a multiple of 2^-24, so is what it is rounded to.
// Growing.  A power of two can take the place of a smaller one without a second rounding of what is above 2^-6 of it; what is below is
// rounded once more, by 2^-10 s each time, 2^-9 s over all times since s at least doubles.
// What is not finite is held as NaN and does not count for the scale.
#pragma once

#include "common.h"

namespace antkv {

constexpr int kScaleRows = 16;
constexpr uint32_t kLeastScale = (127u - 32u) << 23, kMostScale = (127u + 8u) << 23;      // bits of 2^-32, 2^8

// The two halves of four bytes' values x 2^e, e the exponent of `scale`; exact where the product is an fp16 number
__device__ __forceinline__ uint2_t halves_of(uint32_t four, float scale)
{
    return uint2_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, scale, true))};
}
__device__ __forceinline__ half8_t halves_of(uint2_t eight, float scale)
{
    const uint2_t a = halves_of(eight[0], scale), b = halves_of(eight[1], scale);
    return __builtin_bit_cast(half8_t, uint4_t{a[0], a[1], b[0], b[1]});
}

}  // namespace antkv
