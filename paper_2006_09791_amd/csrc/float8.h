// 8-bit float rows: e4m3 values (bias 7, largest 448, no infinities, 0x7f and 0xff not a number) [rows][pitch], pitch = columns rounded up to
// 128 and zeros past the last one, and for each 128 columns a byte [rows][scale pitch]: the exponent, plus 127, of the power of two that
// they are multiplied by.
#pragma once

#include "tokens.h"

namespace gspc {

constexpr int kBlock8 = 128;
__host__ __device__ constexpr int f8_pitch(int cols) { return (cols + kBlock8 - 1) / kBlock8 * kBlock8; }
__host__ __device__ constexpr int f8_scale_pitch(int cols) { return (cols + 4 * kBlock8 - 1) / (4 * kBlock8) * 4; }

// top: the largest finite magnitude of a block.  The smallest power of two with top <= 448 times it, from 2^-127 on (448 = 1.75 2^8).
__device__ __forceinline__ unsigned block_code(unsigned top) {
    const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
    return e > 0 ? e : 0;
}
// What a block's values are multiplied by before they are rounded (a power of two: exact but for what is far below the smallest code).
__device__ __forceinline__ float block_up(unsigned code) { return __uint_as_float((254 - code) << 23); }
// ... and after they are read.  255 stands for no number.
__device__ __forceinline__ float block_down(unsigned code) {
    return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7fc00000u : code << 23);
}
// A magnitude where it is finite, else 0: what is not finite has no say in its block's power of two.
__device__ __forceinline__ unsigned finite_magnitude(float v) {
    const unsigned m = magnitude(v);
    return m < 0x7f800000u ? m : 0u;
}
// Four codes, to nearest, ties to even; infinities and what is no number become no number.
__device__ __forceinline__ unsigned f8_word(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ u32x2 f8_codes(const float (&v)[8], float up) {
    return (u32x2){f8_word(v[0] * up, v[1] * up, v[2] * up, v[3] * up), f8_word(v[4] * up, v[5] * up, v[6] * up, v[7] * up)};
}
__device__ __forceinline__ void f8_values(u32x2 q, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(q[i], true);
        v[4 * i] = lo[0], v[4 * i + 1] = lo[1], v[4 * i + 2] = hi[0], v[4 * i + 3] = hi[1];
    }
}
__device__ __forceinline__ unsigned top_of(const float (&v)[8]) {
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, finite_magnitude(v[e]));
    return top;
}

// Eight columns of a row of which the first n (0 .. 8) are there; the others are 0.
template <typename T> __device__ __forceinline__ Raw<T, 8> fetch_some(const T *p, int n) {
    if (n >= 8) return fetch<8>(p);
    Raw<T, 8> r{};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < n) {
            if constexpr (sizeof(T) == 4) (e < 4 ? r.a : r.b)[e & 3] = p[e];
            else r.a[e / 2] |= (unsigned)p[e] << (e % 2 * 16);
        }
    return r;
}
template <typename T> __device__ __forceinline__ void store_some(T *p, const float (&v)[8], int n, bool past = false) {
    if (n >= 8) store(p, v, past);
    else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) put(p + e, v[e]);
    }
}

}  // namespace gspc
