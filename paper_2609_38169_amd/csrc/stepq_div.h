// Quotients by the constants of FastDiv, in the kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "stepq_layout.h"

namespace stepq {

__device__ __forceinline__ int fdiv(int n, FastDiv d)
{
    const uint32_t u = static_cast<uint32_t>(n);
    return static_cast<int>((__umulhi(u, d.mul) + u) >> d.shift);
}

}  // namespace stepq
