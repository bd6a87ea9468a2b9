// Shared by the calls around the decode step: prompts, single tokens on
// full-precision states, attention over a shared prefix.
#pragma once

#include <stdint.h>
#include <string>
#include <hip/hip_runtime.h>

#include "stepq.h"

namespace stepq {

// Records the calling thread's last failure (stepq_last_error) and returns s.
stepq_status set_error(stepq_status s, const std::string &msg);

inline stepq_status bad(const char *msg) { return set_error(STEPQ_E_INVALID, msg); }

inline stepq_status launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? STEPQ_OK : set_error(STEPQ_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

inline bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline bool known_dtype(int32_t d) { return d == STEPQ_F32 || d == STEPQ_BF16; }

using bf16_t = unsigned short;

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }

// Round to nearest, ties to even; a NaN stays one.
__device__ __forceinline__ bf16_t to_bf16(float x)
{
    return __builtin_bit_cast(bf16_t, static_cast<__bf16>(x));
}

template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16_t narrow<bf16_t>(float x) { return to_bf16(x); }

// alpha or beta, whose type is its own choice (a run-time flag: one value per token and head)
struct Gate {
    const void *p;
    int32_t f32;
    __device__ __forceinline__ float at(size_t i) const
    {
        return f32 ? static_cast<const float *>(p)[i] : widen(static_cast<const bf16_t *>(p)[i]);
    }
};

}  // namespace stepq
