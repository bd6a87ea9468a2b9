// Shared by the attention kernels: reductions over the lanes that hold a query's scores, and the scale's place.
#pragma once

#include "stepq_div.h"
#include "stepq_mma.h"
#include "stepq_plan.h"

namespace stepq {

constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float swap_max16(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float swap_max32(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float swap_add16(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ float swap_add32(float x)
{
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// The scale goes into the exponent, one fma from a score: rounded before the maximum is taken off, scores of 4096
// and more would lose what tells them apart.  That needs it positive (the maximum is taken before): its sign goes
// into the queries, and 0 makes them 0.
__device__ __forceinline__ float scale_of(float scale) { return scale == 0.0f ? 1.0f : fabsf(scale); }
__device__ __forceinline__ u32x4 with_sign(u32x4 q, float scale, uint32_t signs)
{
    return scale > 0.0f ? q : scale == 0.0f ? u32x4{} : q ^ signs;
}

}  // namespace stepq
