// Exponentials, gates and conversions of one value, for kernels that read and write a stream of them.  PRECISE: for binary32 results;
// without it for bfloat16 ones, where a kernel that streams two bytes a value has some ten vector instructions for each and the
// transcendental ones count four times.
#pragma once
#include "common.h"

namespace moe {

constexpr float LOG2E = 1.44269504f, LOG2E_LOW = 1.92596299e-8f, LN2 = 0.693147181f;

// e^x.  The hardware gives 2^y; y = x log2(e) rounded once is off by |x| 2^-24 relative, which a bfloat16 result does not see.  PRECISE
// takes the product's error along: four more operations, off by little more than the hardware's own last bit.
template <bool PRECISE>
__device__ __forceinline__ float exp_of(float x)
{
    const float y = x * LOG2E, e = __builtin_amdgcn_exp2f(y);
    if (!PRECISE) return e;
    const float low = fmaf(x, LOG2E_LOW, fmaf(x, LOG2E, -y));
    // beyond the range the first product is infinite, its error no number
    return fabsf(x) < 126.f ? fmaf(e, low * LN2, e) : e;
}

// A gate's bias as gate_of takes it: without PRECISE -b log2(e), so that the exponent is one multiply-add of the pre-activation.
template <bool PRECISE>
__device__ __forceinline__ float gate_bias(float b) { return PRECISE ? b : -LOG2E * b; }

// s = 1 / (1 + e^-(a + b)) and 1 - s, each with its own relative accuracy (1 - s taken from s would have lost a closed gate's bits).  The exponential
// is kept finite, so that 1 - s is no infinity times zero: s stays at e^-80 or above.  1 - s does reach 0, from a + b = 87 on.  A NaN passes.
template <bool PRECISE>
__device__ __forceinline__ void gate_of(float a, float bias, float &s, float &rest)
{
    float e;
    if (PRECISE) e = exp_of<true>(__builtin_elementwise_minimum(-(a + bias), 80.f));
    else e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(fmaf(a, -LOG2E, bias), 115.4f));
    s = __builtin_amdgcn_rcpf(1.f + e);
    rest = e * s;
}

// tanh c = (1 - a) / (1 + a), a = e^(-2|c|).  1 - a loses bits where c is small: there PRECISE takes the series (up to 0.25, five terms, off by
// 1e-8), a bfloat16 result c itself (up to 0.007: c^2 / 3 and what 1 - a has lost are both below 2e-5).
template <bool PRECISE>
__device__ __forceinline__ float tanh_of(float c)
{
    if (!PRECISE) {
        const float t = fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * LOG2E * c)), 1.f);
        return fabsf(c) < 0.007f ? c : t;
    }
    const float a = exp_of<true>(-2.f * fabsf(c)), c2 = c * c;
    const float t = copysignf((1.f - a) * __builtin_amdgcn_rcpf(1.f + a), c);
    const float series = fmaf(c2, fmaf(c2, fmaf(c2, fmaf(c2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return fabsf(c) < 0.25f ? c * series : t;
}

// with its slope, 1 - tanh^2 c = 4 a / (1 + a)^2: no overflow and no cancellation
template <bool PRECISE>
__device__ __forceinline__ float tanh_of(float c, float &slope)
{
    const float a = exp_of<PRECISE>(-2.f * fabsf(c));
    const float q = __builtin_amdgcn_rcpf(1.f + a);
    slope = a * q * (4.f * q);
    const float t = copysignf((1.f - a) * q, c);
    if (!PRECISE) return fabsf(c) < 0.007f ? c : t;
    const float c2 = c * c;
    const float series = fmaf(c2, fmaf(c2, fmaf(c2, fmaf(c2, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
    return fabsf(c) < 0.25f ? c * series : t;
}

// a stored value as binary32 and back (one rounding)
__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ void store_value(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_value(bf16_t *p, float v) { *p = f32_to_bf16(v); }

}  // namespace moe
