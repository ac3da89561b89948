// Activations, their derivatives and 16-bit packing.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "../../include/som.h"

namespace lay {

// two fp32 values, rounded to nearest even, as one word of two bf16 or fp16
__device__ __forceinline__ uint32_t pack2(float lo, float hi, int bf16)
{
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ float2 unpack2(uint32_t w, int bf16)
{
    if (bf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

__device__ __forceinline__ float unpack1(uint16_t v, int bf16)
{
    if (bf16) return __uint_as_float((uint32_t)v << 16);
    return __half2float(*reinterpret_cast<const __half*>(&v));
}

// eight 16-bit values of a 16-byte word -> fp32
__device__ __forceinline__ void widen8(const uint4& w, float (&v)[8], int bf16)
{
    const float2 a = unpack2(w.x, bf16), b = unpack2(w.y, bf16), c = unpack2(w.z, bf16), d = unpack2(w.w, bf16);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

// the same from memory, 16-byte aligned
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8], int bf16)
{
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    widen8(w, v, bf16);
}

// the largest magnitude, or NaN
__device__ __forceinline__ float largest(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// one instruction each, subnormal results flushed to zero: 2^x off by 2 units, 1 / x by 1 unit in the last place
__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float fast_rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// P(N <= z), and e = exp(-z^2 / 2) that its computation needs: Abramowitz and Stegun 7.1.26 for 1 - erf(|z| / sqrt 2), off by
// at most 1.5e-7, one exponential and one reciprocal for both.  erff and its branch took more time in the epilogues than the
// products left for them.
__device__ __forceinline__ float normal_cdf(float z, float& e)
{
    const float t = fast_rcp(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.f));
    e = fast_exp2(z * (z * -0.72134752f));
    // (the polynomial's coefficients halved)
    const float q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f);
    const float tail = q * e;  // P(N <= -|z|)
    return z < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float sigmoid_of(float z) { return fast_rcp(1.f + fast_exp2(z * -1.44269504f)); }

template <int ACT>
__device__ __forceinline__ float act_of(float z)
{
    if (ACT == SOM_ACT_SILU) return z * sigmoid_of(z);
    if (ACT == SOM_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if (ACT == SOM_ACT_RELU) return z < 0.f ? 0.f : z;
    return z;
}

// the activation and its derivative
template <int ACT>
__device__ __forceinline__ void act_both(float z, float& a, float& da)
{
    if (ACT == SOM_ACT_SILU) {
        const float s = sigmoid_of(z);
        a = z * s;
        da = fmaf(a, 1.f - s, s);
    } else if (ACT == SOM_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        a = z * c;
        da = fmaf(z * 0.39894228f, e, c);
    } else if (ACT == SOM_ACT_RELU) {
        a = z < 0.f ? 0.f : z;
        da = z > 0.f ? 1.f : 0.f;
    } else {
        a = z;
        da = 1.f;
    }
}

template <int ACT>
struct ActTag {
    static constexpr int value = ACT;
};

// f(ActTag) of the activation: the choice is made once for a whole run of values
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    if (act == SOM_ACT_SILU) f(ActTag<SOM_ACT_SILU>());
    else if (act == SOM_ACT_GELU) f(ActTag<SOM_ACT_GELU>());
    else if (act == SOM_ACT_RELU) f(ActTag<SOM_ACT_RELU>());
    else f(ActTag<SOM_ACT_NONE>());
}

}  // namespace lay
