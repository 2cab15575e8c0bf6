// Device side of dropout, for its own kernel and for the residual norms'.
#pragma once

#include <hip/hip_runtime.h>

#include "philox.h"

namespace gspc {

// What columns 8 vec .. 8 vec + 7 of a row are multiplied by: d.up or 0.
__device__ __forceinline__ void dropout_factors(const Dropout &d, uint64_t call, unsigned row, unsigned vec, float (&m)[8]) {
    const Philox p = philox(vec, row, (uint32_t)call, (uint32_t)(call >> 32), d.seed);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        m[2 * e] = (p.word[e] & 0xffffu) >= d.limit ? d.up : 0.f;
        m[2 * e + 1] = p.word[e] >> 16 >= d.limit ? d.up : 0.f;
    }
}

}  // namespace gspc
