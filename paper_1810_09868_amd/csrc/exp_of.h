// Exponentials of differences from a largest score.
#pragma once
#include "common.h"

namespace vgg {

constexpr float kNothing = -1e4f;   // exp of it is 0, and no product with it overflows
// A difference as exp_of takes it: -inf, and what is too low for any exponential, to kNothing; a NaN as it is.
__device__ __forceinline__ float below(float d) { return __builtin_elementwise_maximum(d, kNothing); }
// exp(d), d <= 0 and not below kNothing (or NaN): 2^t, t = d / ln 2 rounded to fp32, times 1 + r, r = d - t ln 2 what that rounding leaves
// (ln 2 in two parts).  Without r a term is off by up to |d| 2^-24, all terms of a flat tail in the same direction.
__device__ __forceinline__ float exp_of(float d)
{
    constexpr float kLog2E = 1.44269504f, kLn2 = 0.693147182f, kLn2Rest = -1.90465421e-9f;
    const float t = d * kLog2E, r = __builtin_fmaf(-t, kLn2Rest, __builtin_fmaf(-t, kLn2, d)), e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, r, e);
}

}  // namespace vgg
