// What the products of 8-bit rows share: loads that are counted and may run past the rows' end, barriers, the order of tiles.
#pragma once

#include "tokens.h"

namespace gspc {

constexpr int kRsrc = 0x00020000;       // raw buffer descriptor: accesses past its end (kOob among them) read zero
constexpr size_t kMostBytes = 1u << 30; // a block's rows are within that: at most 256 of 133152 bytes (integers) or 2^22 (e4m3)

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void *p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)(bytes < kMostBytes ? bytes : kMostBytes), kRsrc);
}

// Waits until at most LEFT of the wave's loads are under way, and for all of its LDS operations.
template <int LEFT> __device__ __forceinline__ void wait_loads() {
    static_assert(LEFT < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4);
}

// Barriers around LDS that loads write directly and other lanes have written: nothing is to be moved across them.  (No fence: that
// would wait for the loads that are to stay under way.)
__device__ __forceinline__ void barrier_of_block() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier_of_wave() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// Workgroups go to the eight XCDs in turn.  Each XCD gets consecutive tiles, and these run through bands of kBand tiles of tokens,
// so that the 32 tiles that an XCD works on together share rows of both operands in its L2.
constexpr unsigned kBand = 8;
__device__ __forceinline__ uint2 tile_of(unsigned mtiles, unsigned ntiles, unsigned b) {
    const unsigned tiles = mtiles * ntiles, each = tiles / 8, more = tiles % 8, xcd = b & 7;
    const unsigned t = xcd * each + min(xcd, more) + (b >> 3);
    const unsigned band = t / (kBand * ntiles), first = band * kBand, high = min(kBand, mtiles - first);
    const unsigned in = t - band * kBand * ntiles;
    return make_uint2(first + in % high, in / high);
}

}  // namespace gspc
