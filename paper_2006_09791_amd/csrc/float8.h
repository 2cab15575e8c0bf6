// 8-bit float rows: e4m3 values (bias 7, largest 448, no infinities, 0x7f and 0xff not a number) [rows][pitch], pitch = columns rounded up to
// 128 and zeros past the last one, and for each 128 columns a byte [rows][scale pitch]: the exponent, plus 127, of the power of two that
// they are multiplied by.
#pragma once

#include "row_place.h"
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
// The largest finite magnitude of some values: what is not finite has no say in its block's power of two.  (The maximum drops what is no number by itself,
// three magnitudes an instruction; values are looked at one by one only where it is an infinity.)
template <int N> __device__ __forceinline__ unsigned top_of(const float (&v)[N]) {
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) top = fmaxf(top, fabsf(v[e]));
    unsigned m = __float_as_uint(top);
    if (m == 0x7f800000u) {
        m = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) m = max(m, magnitude(v[e]) < 0x7f800000u ? magnitude(v[e]) : 0u);
    }
    return m;
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
template <Rows ROWS, bool LONG = false, typename T> __device__ __forceinline__ Raw<T, 8> fetch_some(const T *row, const Place &p) {
    if constexpr (ROWS != kThin) return fetch<8>(beyond(row, column_bytes<LONG>(p.start, sizeof(T))));
    else {
        Raw<T, 8> r{};
#pragma unroll
        for (int e = 0; e < 7; ++e) {
            const T x = row[max(0, min(e, p.n - 1))];
            if constexpr (sizeof(T) == 4) (e < 4 ? r.a : r.b)[e & 3] = x;
            else r.a[e / 2] |= (unsigned)x << (e % 2 * 16);
        }
        return r;
    }
}
// Columns that are not there become 0; all of them do without `there`.
template <Rows ROWS, typename R> __device__ __forceinline__ void widen_some(R raw, const Place &p, float (&v)[8], bool there = true) {
    keep_if(raw, there && p.n > 0);
    widen(raw, v);
    if constexpr (ROWS == kRagged) {
#pragma unroll
        for (int by = 4; by >= 1; by /= 2)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float here = v[e], further = e + by < 8 ? v[(e + by) & 7] : 0.f;
                v[e] = p.shift & by ? further : here;
            }
    }
    if constexpr (ROWS == kThin) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < p.n ? v[e] : 0.f;
    }
}
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *reinterpret_cast<f32x4_any *>(p) = (f32x4){a, b, c, d}; }
__device__ __forceinline__ void store4(uint16_t *p, float a, float b, float c, float d) {
    *reinterpret_cast<u32x2_any *>(p) = (u32x2){bf16_pair(a, b), bf16_pair(c, d)};
}
template <Rows ROWS, bool LONG = false, typename T> __device__ __forceinline__ void store_some(T *row, const Place &p, const float (&v)[8], bool past = false) {
    T *to = beyond(row, column_bytes<LONG>(p.at, sizeof(T)));
    if (p.n == 8) store(to, v, past);
    else if constexpr (ROWS != kWhole) {                 // four, two and one of them (by value: a choice between places would put v into memory)
        const bool four = p.n & 4, two = p.n & 2;
        const float v0 = v[0], v1 = v[1], v2 = v[2], v4 = v[4], v5 = v[5], v6 = v[6];
        const float pair0 = four ? v4 : v0, pair1 = four ? v5 : v1, low = two ? v2 : v0, high = two ? v6 : v4, one = four ? high : low;
        if (four) store4(to, v0, v1, v2, v[3]);
        if (two) {
            put(to + (p.n & 4), pair0);
            put(to + (p.n & 4) + 1, pair1);
        }
        if (p.n & 1) put(to + (p.n & 6), one);
    }
}

}  // namespace gspc
