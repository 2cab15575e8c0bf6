// Dropout's random numbers: Philox 4x32-10 (J. Salmon, M. Moraes, R. Dror, D. Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), ten
// rounds of two products of 32 by 32 bits over a counter of four words.  A number is a function of the seed, the call and the value's place alone,
// so that no mask is stored: the gradient makes it again.  Host and device, without a header of HIP: a test checks it with the host's compiler.
#pragma once

#include <stdint.h>

#include "divide.h"

namespace gspc {

struct Philox {
    uint32_t word[4];
};

GSPC_HD uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);     // (one instruction; of two the compiler makes two)
#else
    return a ^ b ^ c;
#endif
}

GSPC_HD Philox philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint64_t key) {
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
        c1 = (uint32_t)p1;
        c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// Dropout of one call: eight columns share a counter (column / 8, row, the call's number), each has sixteen bits of it.  Values are kept where
// these are no less than `limit` of 65536 (a probability in steps of 2^-16: half the generator's work of 2^-32) and multiplied by `up`.
struct Dropout {
    uint64_t seed, offset;
    const uint64_t *step;       // device memory, added to the offset, or nullptr: what a replayed graph counts on
    uint32_t limit;             // 0: nothing is dropped
    float up;                   // 65536 / (65536 - limit)
};

}  // namespace gspc
