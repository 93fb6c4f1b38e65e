// Rows kept in 8 bits: every kBlock columns of a row share a step, a power of two with which the largest of them has 64 to 127
// steps; a value is kept as the nearest whole number of steps (ties to even, 127 at most).
//
// A power of two, and not a 127th of the largest value: codes and what they stand for are then exact in every type that is narrower
// than 32 bits (7 bits and a sign), so that restored rows are rounded no second time, and a step is one byte.  It costs half a bit
// of resolution on the average.
#pragma once
#include "dense.hpp"

namespace nacho {

constexpr int kBlock = 32;             // columns that share a step

// The step's exponent as it is stored (127 added; 0: also of smaller ones), from the bits of the largest magnitude of a block; 255: it has a
// NaN or an infinity, and all of it is restored as NaN.
__device__ inline unsigned exponent_of(unsigned most)
{
    const unsigned e = most >> 23;
    return e == 255 ? 255u : e > 6 ? e - 6 : 0u;
}
// What values are multiplied by to be steps.
__device__ inline float steps_per(unsigned exponent) { return exponent == 255 ? 0.0f : __uint_as_float((254 - exponent) << 23); }
// A step.
__device__ inline float step_of(unsigned exponent)
{
    return __uint_as_float(exponent == 255 ? 0x7fc00000u : exponent == 0 ? 0x00400000u : exponent << 23);
}
__device__ inline unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Four codes of finite values.  (The sum with 3 x 2^22 rounds to whole numbers, and ends in their lowest byte.)
__device__ inline unsigned four_codes(float a, float b, float c, float d, float by)
{
    auto code = [&](float v) { return __float_as_uint(__builtin_amdgcn_fmed3f(__builtin_fmaf(v, by, 12582912.0f), 12582785.0f, 12583039.0f)); };
    const unsigned low = __builtin_amdgcn_perm(code(b), code(a), 0x0c0c0400u), high = __builtin_amdgcn_perm(code(d), code(c), 0x04000c0cu);
    return low | high;
}
// The value of code number i of four.
__device__ inline float value_of(unsigned codes, int i, float step) { return (float)((int)(codes << (24 - 8 * i)) >> 24) * step; }

}  // namespace nacho
