// Activations between the layers of a mixture of experts, and their slopes.
#pragma once
#include "dense.hpp"

namespace nacho {

// Activations and their slopes.  Rows of floats take the library's functions, and slopes in 64 bits: next to its root a
// slope is a difference of nearly equal numbers.  For rows of 16 bits the normal distribution comes from a polynomial (in the
// form of Abramowitz and Stegun 7.1.26, fitted here): erfc(x) exp(x^2) = t P(t) with t = 1 / (1 + 0.38 x), relative error below
// 4e-7 for all x >= 0 in 32 bits, a hundredth of what the rounding to the type takes; and it shares its exponential with the
// density.  (16384 x 4096 bf16, slopes of gelu: 143 us with erfcf, bound by its instructions.)
struct Normal {
    float below, density;
    __device__ explicit Normal(float z)
    {
        const float t = __builtin_amdgcn_rcpf(1.0f + 2.687005769e-01f * fabsf(z)), e = exp2_of(-0.5f * kLog2e * z * z);
        const float c[9] = {2.144118706e-01f, 2.139049757e-01f, 2.040023426e-01f, 1.382982534e-01f, 2.308058125e-01f,
                            -1.625332754e-01f, 3.647579072e-01f, -2.626970734e-01f, 5.904920688e-02f};
        float p = c[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = p * t + c[i];
        const float tail = 0.5f * t * p * e;
        below = z < 0.0f ? tail : 1.0f - tail;
        density = 0.3989422804014327f * e;
    }
};
template <typename T> __device__ inline float activated(float z, int act)
{
    if (act == NACHO_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
    if (act == NACHO_ACT_GELU) {
        // (by the complement of the error function: next to one, 1 + erf has no digits left for a negative argument)
        if constexpr (sizeof(T) == 4) return z * 0.5f * erfcf(-0.70710678118654752f * z);
        else return z * Normal(z).below;
    }
    if (act == NACHO_ACT_SILU) {
        if constexpr (sizeof(T) == 4) return z / (1.0f + expf(-z));
        else return z * __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * z));
    }
    return z;
}
// (A row past its type's range is kept as an infinity: its slope is that of any number so far out, 0 or 1, where the formulas'
// products of zero and infinity would make a NaN.)
template <typename T> __device__ inline float slope_at(float z, int act)
{
    if (act == NACHO_ACT_RELU) return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
    if constexpr (sizeof(T) == 4) {
        const double v = z;
        if (act == NACHO_ACT_GELU) {
            const double density = 0.39894228040143267794 * exp(-0.5 * v * v);
            return (float)(0.5 * erfc(-0.70710678118654752440 * v) + (density == 0.0 ? 0.0 : v * density));
        }
        if (act == NACHO_ACT_SILU) {
            const double q = 1.0 / (1.0 + exp(-v)), both = q * (1.0 - q);
            return (float)(both == 0.0 ? q : q + v * both);
        }
    } else {
        if (act == NACHO_ACT_GELU) {
            const Normal at(z);
            return at.below + (at.density == 0.0f ? 0.0f : z * at.density);
        }
        if (act == NACHO_ACT_SILU) {
            const float q = __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * z)), both = q * (1.0f - q);
            return both == 0.0f ? q : q + z * both;
        }
    }
    return 1.0f;
}

}  // namespace nacho
