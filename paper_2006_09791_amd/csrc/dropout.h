// Device side of dropout, for its own kernel and for the residual norms'.
#pragma once

#include <hip/hip_runtime.h>

#include "philox.h"

namespace gspc {

// The numbers of columns 8 vec .. 8 vec + 7 of a row.
__device__ __forceinline__ Philox drop_numbers(const Dropout &d, uint64_t call, unsigned row, unsigned vec) {
    return philox(vec, row, (uint32_t)call, (uint32_t)(call >> 32), d.seed);
}
// Values of columns that are dropped become 0, whatever they are.
__device__ __forceinline__ void drop_by(const Philox &p, uint32_t limit, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = (p.word[e] & 0xffffu) >= limit ? v[2 * e] : 0.f;
        v[2 * e + 1] = p.word[e] >> 16 >= limit ? v[2 * e + 1] : 0.f;
    }
}
__device__ __forceinline__ void drop_some(const Dropout &d, uint64_t call, unsigned row, unsigned vec, float (&v)[8]) {
    drop_by(drop_numbers(d, call, row, vec), d.limit, v);
}

}  // namespace gspc
