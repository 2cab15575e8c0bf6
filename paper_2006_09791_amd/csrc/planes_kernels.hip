// NCHW planes to channels-last tokens and back: the transpose of [R][S] to [S][R] in every image, with a change of type.
#include "tokens.h"
#include "tokens_internal.h"

namespace gspc {

constexpr int kTile = 64, kTilePitch = kTile + 1;

// One block transposes a 64 x 64 tile through LDS in fp32; the last tiles of a row or column are moved back so that they end
// with it (what they share with their neighbours is written twice, the same), so that only planes smaller than a tile have
// lanes without work.  VI, VO: elements per access along S and along R: 8, or 1 where both sides have fewer than 8.
// The pitch of 65 words puts the 64 words that a wave writes (8 rows x 8 vectors, one element of each) and reads (the same
// the other way) into 64 banks.  Bound by memory: each element is read and written once; 256 images of
// 128 x 784 from fp32 to bf16 26.6 us, 5.8 TB/s, what a large copy reaches and more.
template <typename TI, typename TO, int VI, int VO>
__global__ __launch_bounds__(256) void transpose_kernel(const TI *__restrict__ in, TO *__restrict__ out, int R, int S, unsigned rtiles,
                                                       unsigned tiles, unsigned m_rtiles, unsigned m_tiles, int past, unsigned first) {
    __shared__ float lds[kTile * kTilePitch];
    const unsigned b = first + blockIdx.x, n = fast_div_any(b, tiles, m_tiles), t = b - n * tiles;
    const unsigned st = fast_div_any(t, rtiles, m_rtiles), rt = t - st * rtiles;
    const int wr = min(R, kTile), ws = min(S, kTile);
    const int r0 = min((int)rt * kTile, R - wr), s0 = min((int)st * kTile, S - ws);
    const TI *ip = in + (size_t)n * R * S + (size_t)r0 * S + s0;
    TO *op = out + (size_t)n * R * S + (size_t)s0 * R + r0;
    Raw<TI, VI> raw[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * 256 + threadIdx.x, r = i >> 3, at = vector_start<VI>(i & 7, ws);
        if (r < wr && (i & 7) < vectors_of<VI>(ws)) raw[k] = fetch<VI>(ip + (size_t)r * S + at);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * 256 + threadIdx.x, r = i >> 3, at = vector_start<VI>(i & 7, ws);
        if (r < wr && (i & 7) < vectors_of<VI>(ws)) {
            float v[VI];
            widen(raw[k], v);
#pragma unroll
            for (int e = 0; e < VI; ++e) lds[(at + e) * kTilePitch + r] = v[e];
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = k * 256 + threadIdx.x, s = i >> 3, at = vector_start<VO>(i & 7, wr);
        if (s < ws && (i & 7) < vectors_of<VO>(wr)) {
            float v[VO];
#pragma unroll
            for (int e = 0; e < VO; ++e) v[e] = lds[s * kTilePitch + at + e];
            store(op + (size_t)s * R + at, v, past);
        }
    }
}

// One side of fewer than 8 (a network's first image): kLong of the other side at a time, where one of the two tensors is one piece of
// memory.  THIN_IN: the input is [R][S < 8], that piece; else it is [R < 8][S] and the output is.
constexpr int kLong = 1024;
template <typename TI, typename TO, bool THIN_IN>
__global__ __launch_bounds__(256) void transpose_thin_kernel(const TI *__restrict__ in, TO *__restrict__ out, int thin, int wide, unsigned tiles,
                                                            unsigned m_tiles, unsigned m_thin, int past) {
    __shared__ float lds[kLong * 7];                // [long][thin]
    const unsigned n = fast_div_any(blockIdx.x, tiles, m_tiles), t = blockIdx.x - n * tiles;
    const int w = min(wide, kLong), l0 = min((int)t * kLong, wide - w);
    const size_t image = (size_t)n * thin * wide;
    // the piece [w][thin]
    const auto piece = [&](auto body) {
        const int count = w * thin;
        for (int i = threadIdx.x; i < (count + 7) / 8; i += 256) body(min(i * 8, count - 8));
    };
    // its columns, `vectors` of each
    const auto columns = [&](auto body) {
        const int vectors = (w + 7) / 8;
        for (int i = threadIdx.x; i < vectors * thin; i += 256) {
            const int v = fast_div(i, m_thin);
            body(i - v * thin, min(v * 8, w - 8));
        }
    };
    if constexpr (THIN_IN) {
        piece([&](int at) {
            float v[8];
            widen(fetch<8>(in + image + (size_t)l0 * thin + at), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[at + e] = v[e];
        });
    } else {
        columns([&](int c, int at) {
            float v[8];
            widen(fetch<8>(in + image + (size_t)c * wide + l0 + at), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[(at + e) * thin + c] = v[e];
        });
    }
    __syncthreads();
    if constexpr (THIN_IN) {
        columns([&](int c, int at) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = lds[(at + e) * thin + c];
            store(out + image + (size_t)c * wide + l0 + at, v, past);
        });
    } else {
        piece([&](int at) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = lds[at + e];
            store(out + image + (size_t)l0 * thin + at, v, past);
        });
    }
}

// Launches for N images of `tiles` blocks each: f(first image, first tile, blocks).
template <typename F> static void in_launches(int N, unsigned tiles, unsigned threads, const F &f) {
    const unsigned most = most_blocks(threads);
    const long step = tiles > most ? 1 : most / tiles;
    for (long n = 0; n < N; n += step) {
        const unsigned all = tiles * (unsigned)(N - n < step ? N - n : step);      // more than a launch may have: of one image
        for (unsigned first = 0; first < all; first += most) f((size_t)n, first, all - first < most ? all - first : most);
    }
}

template <typename TI, typename TO>
static hipError_t transpose(const void *in, int N, int R, int S, void *out, hipStream_t s) {
    const bool large = sizeof(TO) == 2 && (size_t)N * R * S * 2 >= kPastCaches, whole = whole_pieces(out, (size_t)R * 2, (size_t)R * 2);
    if ((R < 8) != (S < 8)) {                       // 152 images of 6 x 10954 in bf16: 17.8 us in tiles of 64 x 64
        const int thin = R < S ? R : S, wide = R < S ? S : R;
        const unsigned tiles = (wide - 1) / kLong + 1;
        const int past = large && (R < S || whole);             // (images of one piece, or R values at a time)
        const auto kern = S < R ? transpose_thin_kernel<TI, TO, true> : transpose_thin_kernel<TI, TO, false>;
        in_launches(N, tiles, 256, [&](size_t n, unsigned, unsigned blocks) {      // (an image is at most 2^21 tiles)
            hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, s, static_cast<const TI *>(in) + n * R * S,
                               static_cast<TO *>(out) + n * R * S, thin, wide, tiles, div_magic(tiles), div_magic(thin), past);
        });
        return hipGetLastError();
    }
    const unsigned rt = (R - 1) / kTile + 1, st = (S - 1) / kTile + 1;
    const unsigned tiles = rt * st;
    // Past the caches: 256 images of 128 x 784 in bf16 to tokens (256 bytes each) 22.0 us through them and 21.4 past; back (1568 bytes) 18.6 and 24.0.
    const int past = large && whole && R >= kTile;
    const auto kern = R >= 8 ? transpose_kernel<TI, TO, 8, 8> : transpose_kernel<TI, TO, 1, 1>;
    in_launches(N, tiles, 256, [&](size_t n, unsigned first, unsigned blocks) {
        hipLaunchKernelGGL(kern, dim3(blocks), dim3(256), 0, s, static_cast<const TI *>(in) + n * R * S,
                           static_cast<TO *>(out) + n * R * S, R, S, rt, tiles, div_magic(rt), div_magic(tiles), past, first);
    });
    return hipGetLastError();
}

hipError_t launch_transpose(const void *in, int in_dtype, int N, int R, int S, void *out, int out_dtype, hipStream_t s) {
    if (in_dtype == GSPC_F32)
        return out_dtype == GSPC_F32 ? transpose<float, float>(in, N, R, S, out, s) : transpose<float, uint16_t>(in, N, R, S, out, s);
    return out_dtype == GSPC_F32 ? transpose<uint16_t, float>(in, N, R, S, out, s) : transpose<uint16_t, uint16_t>(in, N, R, S, out, s);
}

}  // namespace gspc
