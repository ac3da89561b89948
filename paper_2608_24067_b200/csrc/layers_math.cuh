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

// eight consecutive 16-bit values, 16-byte aligned
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8], int bf16)
{
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
    const float2 a = unpack2(w.x, bf16), b = unpack2(w.y, bf16), c = unpack2(w.z, bf16), d = unpack2(w.w, bf16);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
}

__device__ __forceinline__ float act_of(float z, int act)
{
    if (act == SOM_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));
    if (act == SOM_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    if (act == SOM_ACT_RELU) return z < 0.f ? 0.f : z;
    return z;
}

// the activation and its derivative
__device__ __forceinline__ void act_both(float z, int act, float& a, float& da)
{
    if (act == SOM_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        a = z * s;
        da = s * (1.f + z * (1.f - s));
    } else if (act == SOM_ACT_GELU) {
        const float c = 0.5f * (1.f + erff(z * 0.70710678118654752f));
        a = z * c;
        da = c + z * 0.39894228040143268f * __expf(-0.5f * z * z);
    } else if (act == SOM_ACT_RELU) {
        a = z < 0.f ? 0.f : z;
        da = z > 0.f ? 1.f : 0.f;
    } else {
        a = z;
        da = 1.f;
    }
}

}  // namespace lay
