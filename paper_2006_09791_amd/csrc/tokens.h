// Device helpers of the channels-last operators: eight consecutive channels of one token at a time, whatever their type.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "divide.h"

namespace gspc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Rows of any stride start at any multiple of their element's size: vector accesses that ask for no more than that.  (The
// hardware takes them; a 16-byte access that straddles two cache lines costs a second one.)
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef u32x2 __attribute__((aligned(1))) u32x2_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

constexpr int kWave = 64;

__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {   // to nearest, ties to even; NaN stays one
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(unsigned, (bf16x2){(__bf16)lo, (__bf16)hi});
}
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// Storage types: float, uint16_t (bf16) and int8_t (the values of 8-bit rows, without their scale).
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(uint16_t v) { return __uint_as_float((unsigned)v << 16); }
__device__ __forceinline__ float as_float(int8_t v) { return (float)v; }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = to_bf16(v); }

// V = 8: a vector; V = 1: a single element (rows of fewer than eight channels).
struct Raw32 { f32x4 a, b; };
struct Raw16 { u32x4 a; };
struct Raw8 { u32x2 a; };
template <typename T, int V> struct RawOf { typedef T type; };
template <> struct RawOf<float, 8> { typedef Raw32 type; };
template <> struct RawOf<uint16_t, 8> { typedef Raw16 type; };
template <> struct RawOf<int8_t, 8> { typedef Raw8 type; };
template <typename T, int V> using Raw = typename RawOf<T, V>::type;

// Element `off` bytes beyond an address that is the same for the whole wave: the form that needs one register of address.
template <typename T> __device__ __forceinline__ T *beyond(T *base, unsigned off) {
    typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte;
    return reinterpret_cast<T *>(reinterpret_cast<byte *>(base) + off);
}

// Loads stay raw until they are used, so that several can be in flight.
template <int V> __device__ __forceinline__ Raw<float, V> fetch(const float *p) {
    if constexpr (V == 1) return *p;
    else return {*reinterpret_cast<const f32x4_any *>(p), *reinterpret_cast<const f32x4_any *>(p + 4)};
}
template <int V> __device__ __forceinline__ Raw<uint16_t, V> fetch(const uint16_t *p) {
    if constexpr (V == 1) return *p;
    else return {*reinterpret_cast<const u32x4_any *>(p)};
}
template <int V> __device__ __forceinline__ Raw<int8_t, V> fetch(const int8_t *p) {
    if constexpr (V == 1) return *p;
    else return {*reinterpret_cast<const u32x2_any *>(p)};
}
// Nothing computed from r before is used after: values that are held raw over several passes are widened anew in each (kept
// wide they would take twice the registers).
__device__ __forceinline__ void hold(Raw32 &r) { asm volatile("" : "+v"(r.a), "+v"(r.b)); }
__device__ __forceinline__ void hold(Raw16 &r) { asm volatile("" : "+v"(r.a)); }
__device__ __forceinline__ void hold(Raw8 &r) { asm volatile("" : "+v"(r.a)); }
template <typename T> __device__ __forceinline__ void hold(T &) {}

__device__ __forceinline__ void keep_if(Raw32 &r, bool yes) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.a[e] = yes ? r.a[e] : 0.f, r.b[e] = yes ? r.b[e] : 0.f;
}
__device__ __forceinline__ void keep_if(Raw16 &r, bool yes) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.a[e] = yes ? r.a[e] : 0u;
}
template <typename T> __device__ __forceinline__ void keep_if(T &r, bool yes) { r = yes ? r : T(0); }

__device__ __forceinline__ void widen(const Raw32 &r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = r.a[e], v[4 + e] = r.b[e];
}
__device__ __forceinline__ void widen(const Raw16 &r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(r.a[e] << 16), v[2 * e + 1] = __uint_as_float(r.a[e] & 0xffff0000u);
}
__device__ __forceinline__ void widen(const Raw8 &r, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(r.a[e / 4] >> (e % 4 * 8));
}
template <typename T> __device__ __forceinline__ void widen(const T &r, float (&v)[1]) { v[0] = as_float(r); }

// past: beyond the caches (a non-temporal store), for outputs of kPastCaches bytes and more in bf16.  Group norm in bf16, us alone and with a
// reader of y behind it: 12.8 MB of y 10.6 and 15.6 through the caches, 9.4 and 14.9 past them; 25.7 MB 13.8, 22.4 and 12.2, 21.7; 51 MB
// 29.5, 43.1 and 19.2, 46.0; below 8 MB level.
// Only whole pieces of 64 bytes, or what lies side by side: 64 images of 56x56, 40 of 160 channels 16.4 through the caches and 22.5 past
// them, 100 of 200 38.1 and 44.3, 64 of 128 20.3 and 18.0, 40 of 40 15.4 and 13.9.
constexpr size_t kPastCaches = 8u << 20;
// Whether rows of `bytes` bytes, `ld` bytes apart, from p on are whole pieces.
inline bool whole_pieces(const void *p, size_t bytes, size_t ld) { return (reinterpret_cast<uintptr_t>(p) | bytes | ld) % 64 == 0; }
// (two stores that differ in their hint alone would be merged, without the empty statements)
__device__ __forceinline__ void store_vector(u32x4_any *p, u32x4 v, bool past) {
    if (past) {
        asm volatile("");
        __builtin_nontemporal_store((u32x4_any)v, p);
        asm volatile("");
    } else
        *p = v;
}
// (fp32 through the caches always: two stores of 16 bytes of every 32 are no whole pieces.  64 images of 56x56, group norm with 96 channels side
// by side 43.7 us and 55.2 past the caches, 128 of 28x28 with 48 11.7 and 20.2.)
__device__ __forceinline__ void store(float *p, const float (&v)[8], bool = false) {
    *reinterpret_cast<f32x4_any *>(p) = (f32x4){v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any *>(p + 4) = (f32x4){v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store(uint16_t *p, const float (&v)[8], bool past = false) {
    const u32x4 r = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    store_vector(reinterpret_cast<u32x4_any *>(p), r, past);
}
template <typename T> __device__ __forceinline__ void store(T *p, const float (&v)[1], bool = false) { put(p, v[0]); }

// A row of C channels in vectors of V: vector i starts at channel 8 i, the last one at C - 8, so that it ends with the row.
// Its first overlap(i) channels belong to the vector before it too: both write them, with the same values, and sums over
// channels leave them out here.
template <int V> __device__ __forceinline__ int vector_start(int i, int C) { return V == 1 ? i : min(i * V, C - V); }
template <int V> __host__ __device__ __forceinline__ int vectors_of(int C) { return (C + V - 1) / V; }

// A reduction over groups of `width` lanes (a power of two, the same for the whole wave); every lane gets its group's result.
// Within 16 lanes by DPP operands, beyond by the row swaps: a step is two instructions without a trip through LDS.
template <typename T, typename F> __device__ __forceinline__ T lanes_reduce(T v, int width, const F &f) {
    const auto dpp = [](T x, auto ctrl) {
        return __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if (width >= 2) v = f(v, dpp(v, std::integral_constant<int, 0xb1>{}));      // quad_perm: lane ^ 1
    if (width >= 4) v = f(v, dpp(v, std::integral_constant<int, 0x4e>{}));      // quad_perm: lane ^ 2
    if (width >= 8) v = f(v, dpp(v, std::integral_constant<int, 0x141>{}));     // row_half_mirror: the other four of eight
    if (width >= 16) v = f(v, dpp(v, std::integral_constant<int, 0x140>{}));    // row_mirror: the other eight of a row
    if (width >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);    // the other row of two
        v = f(__builtin_bit_cast(T, (unsigned)r[0]), __builtin_bit_cast(T, (unsigned)r[1]));
    }
    if (width >= 64) {
        const unsigned u = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);    // the other half of the wave
        v = f(__builtin_bit_cast(T, (unsigned)r[0]), __builtin_bit_cast(T, (unsigned)r[1]));
    }
    return v;
}
__device__ __forceinline__ float lanes_sum(float v, int width) {
    return lanes_reduce(v, width, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ unsigned lanes_umax(unsigned v, int width) {
    return lanes_reduce(v, width, [](unsigned a, unsigned b) { return max(a, b); });
}

// ---- 8-bit rows: q = rint(x * (127 / a)) to even, a = max |x| of the row; x is read back as q * (a / 127) ------------------
__host__ __device__ constexpr int rows8_pitch(int cols) { return (cols + 15) / 16 * 16; }

// |v| as a number that orders like an integer, infinity above every finite value and NaN above infinity: one maximum over a
// row says how large it is and whether all of it is finite.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct RowCode {
    float up, inv, scale;
    unsigned keep;
};
// top: the largest magnitude of the row.  A row that is not finite gets the scale NaN and zeros, so that all of it is read back
// as NaN.  A row below 2^-64 is coded 2^64 times larger: 127 / a would overflow.
__device__ __forceinline__ RowCode row_code(unsigned top) {
    const float a = __uint_as_float(top);
    RowCode c;
    c.keep = top < 0x7f800000u ? 0xffffffffu : 0u;
    c.up = a < 0x1p-64f ? 0x1p64f : 1.f;
    c.inv = top ? 127.f / (a * c.up) : 0.f;
    c.scale = c.keep ? a / 127.f : __uint_as_float(0x7fc00000u);
    return c;
}
// The low byte of the result is the code: adding 1.5 * 2^23 rounds to whole numbers, ties to even.  (Two products and a sum,
// each rounded: contracted to one operation they would round other values than the definition's.)
__device__ __forceinline__ unsigned code_bits(float v, const RowCode &c) {
#pragma clang fp contract(off)
    const float t = v * c.up * c.inv;
    return __float_as_uint(t + 12582912.f);
}
__device__ __forceinline__ unsigned code_word(float v0, float v1, float v2, float v3, const RowCode &c) {
    const unsigned lo = __builtin_amdgcn_perm(code_bits(v1, c), code_bits(v0, c), 0x0c0c0400u);
    const unsigned hi = __builtin_amdgcn_perm(code_bits(v3, c), code_bits(v2, c), 0x04000c0cu);
    return (lo | hi) & c.keep;
}
// (Through the caches, whatever the size: rows that a norm saves, 256 images of 28x28, 128 channels, 36.6 us and 35.4 past them, and with the gradient
// that reads them 78.8 and 81.0; in fp32 112 and 123.)
__device__ __forceinline__ void store_codes(int8_t *p, const float (&v)[8], const RowCode &c) {
    *reinterpret_cast<u32x2_any *>(p) = (u32x2){code_word(v[0], v[1], v[2], v[3], c), code_word(v[4], v[5], v[6], v[7], c)};
}
__device__ __forceinline__ void store_codes(int8_t *p, const float (&v)[1], const RowCode &c) { *p = (int8_t)(code_bits(v[0], c) & c.keep); }

// ---- activations ------------------------------------------------------------------------------------------------------------
enum { kActNone = 0, kActRelu = 1, kActSilu = 2 };

// 1 / (1 + e^-z) by the hardware's 2^x and reciprocal (each within an ulp).  The rounding of z log2(e) is an error of |z| 2^-24
// of e^-z: for z >= 0 less than an ulp of the result, for negative z as much of the result itself (2e-7 at -3, 1e-6 at -17, 5e-6 at -85; never
// above 2e-8 in absolute terms).
__device__ __forceinline__ float sigmoid(float z) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}
template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == kActRelu) return z < 0.f ? 0.f : z;      // NaN stays one
    if constexpr (ACT == kActSilu) return z * sigmoid(z);
    return z;
}
// act'(z); ReLU's at 0 is 0.
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == kActRelu) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if constexpr (ACT == kActSilu) {
        const float s = sigmoid(z);
        return fmaf(s, fmaf(-s, z, z), s);                        // s + s z (1 - s)
    }
    return 1.f;
}

}  // namespace gspc
