// What the kernels of the cross entropy share.
#pragma once
#include "products.hpp"

namespace nacho {

// For f16: the power of two that brings the largest weight of a row next to 2^15.  The products of a gradient read g times it: the small
// probabilities of most of a vocabulary, under weights of one by the number of rows, would vanish.
__device__ inline int scale_exponent(float most)
{
    const int e = most > 0.0f && most < kInfinity ? 14 - ilogbf(most) : 0;
    return e < 100 ? e : 100;
}

}  // namespace nacho
