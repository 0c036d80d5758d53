// Exponentials, gates and conversions of one value, for kernels that read and write a stream of them.
#pragma once
#include "common.h"

namespace moe {

// e^x.  The hardware gives 2^y; y = x log2(e) rounded once is off by |x| 2^-24 relative, which a bfloat16 result does not see.  PRECISE
// (binary32 results) takes the product's error along: four more operations, off by little more than the hardware's own last bit.
template <bool PRECISE>
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float LOG2E = 1.44269504f, LOG2E_LOW = 1.92596299e-8f, LN2 = 0.693147181f;
    const float y = x * LOG2E, e = __builtin_amdgcn_exp2f(y);
    if (!PRECISE) return e;
    const float low = fmaf(x, LOG2E_LOW, fmaf(x, LOG2E, -y));
    // beyond the range the first product is infinite, its error no number
    return fabsf(x) < 126.f ? fmaf(e, low * LN2, e) : e;
}

// s = 1 / (1 + e^-z) and 1 - s, each with its own relative accuracy (1 - s taken from s would have lost a closed gate's bits).  e^-z is kept
// finite, so that the second is no infinity times zero; a NaN passes.
template <bool PRECISE>
__device__ __forceinline__ void gate_of(float z, float &s, float &rest)
{
    const float e = exp_of<PRECISE>(z < -80.f ? 80.f : -z);
    s = __builtin_amdgcn_rcpf(1.f + e);
    rest = e * s;
}

// tanh c, and 1 - tanh^2 c = 4 a / (1 + a)^2 with a = e^(-2|c|): no overflow and no cancellation.  Small arguments take the series, since
// 1 - a loses bits there: up to |c| = 0.25 with five terms, off by 1e-8 (PRECISE), up to 0.06 with two, off by 2e-6.
template <bool PRECISE>
__device__ __forceinline__ float tanh_of(float c, float &slope)
{
    const float a = exp_of<PRECISE>(-2.f * fabsf(c));
    const float q = __builtin_amdgcn_rcpf(1.f + a);
    const float t = copysignf((1.f - a) * q, c), c2 = c * c;
    slope = 4.f * a * (q * q);
    const float series = PRECISE ? fmaf(c2, fmaf(c2, fmaf(c2, fmaf(c2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f)
                                 : fmaf(c2, -1.f / 3.f, 1.f);
    return fabsf(c) < (PRECISE ? 0.25f : 0.06f) ? c * series : t;
}

// a stored value as binary32 and back (one rounding)
__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(bf16_t *p, float v) { *p = f32_to_bf16(v); }

}  // namespace moe
