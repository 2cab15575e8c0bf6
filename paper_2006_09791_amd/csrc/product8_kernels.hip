// out[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k] + bias[n], a and w 8-bit rows: integer sums on the matrix cores, exact.
#include "tokens.h"
#include "tokens_internal.h"

namespace gspc {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kRsrc = 0x00020000;       // raw buffer descriptor: accesses past its end (kOob among them) read zero
constexpr size_t kMostBytes = 1u << 30; // a block's rows are within that: at most 256 of 133152 bytes

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void *p, size_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)(bytes < kMostBytes ? bytes : kMostBytes), kRsrc);
}

struct ProductArgs {
    const int8_t *a, *w;
    const float *a_scale, *w_scale, *bias;
    void *out;
    size_t M, ldo;
    int N, pitch;
    unsigned mtiles, ntiles;
};

// Four consecutive outputs of one token.
template <typename T>
__device__ __forceinline__ void put4(const ProductArgs &p, size_t m, int n, const float (&v)[4]) {
    T *o = static_cast<T *>(p.out) + m * p.ldo + n;
    if (n + 3 < p.N) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_any *>(o) = (f32x4){v[0], v[1], v[2], v[3]};
        else *reinterpret_cast<u32x2_any *>(o) = (u32x2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) put(o + e, v[e]);
    }
}
__device__ __forceinline__ void channel_terms(const ProductArgs &p, int n, float (&scale)[4], float (&bias)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int c = min(n + e, p.N - 1);
        scale[e] = p.w_scale[c];
        bias[e] = p.bias ? p.bias[c] : 0.f;
    }
}

// ---- few tokens or few outputs: no staging --------------------------------------------------------------------------------------
// A block has 16 TN channels x 16 TM tokens; its waves take k-steps of 64 in turn, operands straight from memory into the
// registers of v_mfma_i32_16x16x64_i8 (channels are the rows, tokens the columns of its result), and join their sums in LDS.
template <typename T, int TN, int TM, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product8_small_kernel(ProductArgs p) {
    __shared__ i32x4 s_part[WAVES][TN * TM][kWave];
    const unsigned nt = blockIdx.x % p.ntiles, mt = blockIdx.x / p.ntiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n0 = nt * 16 * TN;
    const size_t m0 = (size_t)mt * 16 * TM;
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const unsigned row = lane % 16, col = lane / 16 * 16;
    i32x4 acc[TN][TM] = {};
    for (int k = wave * 64; k < p.pitch; k += WAVES * 64) {
        const unsigned at = row * p.pitch + k + col;
        const bool in = k + (int)col < p.pitch;
        i32x4 w[TN], a[TM];
#pragma unroll
        for (int i = 0; i < TN; ++i)
            w[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, in ? at + i * 16 * p.pitch : kOob, 0, 0));
#pragma unroll
        for (int j = 0; j < TM; ++j)
            a[j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, in ? at + j * 16 * p.pitch : kOob, 0, 0));
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], a[j], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) s_part[wave][i * TM + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = threadIdx.x; t < TN * TM * kWave; t += 64 * WAVES) {
        const int tile = t / kWave, l = t % kWave;
        i32x4 sum = s_part[0][tile][l];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += s_part[v][tile][l];
        const size_t m = m0 + tile % TM * 16 + l % 16;
        const int n = n0 + tile / TM * 16 + l / 16 * 4;
        if (m < p.M && n < p.N) {
            float scale[4], bias[4], v[4];
            channel_terms(p, n, scale, bias);
            const float sa = p.a_scale[m];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (float)sum[e] * sa * scale[e] + bias[e];
            put4<T>(p, m, n, v);
        }
    }
}

// ---- many tokens: tiles through LDS ---------------------------------------------------------------------------------------------
constexpr int kStep = 128;              // bytes of a row that one stage holds

// WM x WN waves of TM x TN products 32x32x32 each.  A stage holds 128 bytes of BM + BN rows, brought by loads that write LDS
// directly (16 bytes a lane, eight rows a wave), while the other stage is multiplied.  Within a row the 16-byte pieces are
// permuted by the row's number, so that the lanes that read one column of pieces spread over all banks; a load's lanes fetch
// from the addresses that this asks for.
template <typename T, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN) void product8_tile_kernel(ProductArgs p) {
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, ROWS = BM + BN, LOADS = ROWS / 8 / WAVES;
    static_assert(ROWS % (8 * WAVES) == 0, "whole loads");
    __shared__ char stage0[ROWS * kStep], stage1[ROWS * kStep];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const unsigned mt = blockIdx.x / p.ntiles, nt = blockIdx.x % p.ntiles;
    const size_t m0 = (size_t)mt * BM;
    const int n0 = nt * BN;
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const auto swizzle = [](int row) { return (row & 7) ^ (row >> 3 & 1); };

    const auto load = [&](char *stage, int k) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int base = (i * WAVES + wave) * 8, row = base + lane / 8, piece = (lane % 8) ^ swizzle(row);
            const int at = k + piece * 16;
            const bool tokens = base < BM;
            const unsigned off = at < p.pitch ? (unsigned)(tokens ? row : row - BM) * p.pitch + at : kOob;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(tokens ? ra : rw, (__attribute__((address_space(3))) void *)(stage + base * kStep), 16,
                                                     off, 0, 0, 0);
        }
    };
    i32x16 acc[TM][TN] = {};
    const int wm = wave / WN * TM * 32, wn = BM + wave % WN * TN * 32, r = lane % 32, half = lane / 32;
    const auto multiply = [&](const char *stage) {
#pragma unroll
        for (int k = 0; k < kStep / 32; ++k) {
            i32x4 a[TM], w[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i)
                a[i] = *reinterpret_cast<const i32x4 *>(stage + (wm + i * 32 + r) * kStep + (((2 * k + half) ^ swizzle(r)) * 16));
#pragma unroll
            for (int j = 0; j < TN; ++j)
                w[j] = *reinterpret_cast<const i32x4 *>(stage + (wn + j * 32 + r) * kStep + (((2 * k + half) ^ swizzle(r)) * 16));
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[j], a[i], acc[i][j], 0, 0, 0);
        }
    };
    const auto wait = [] {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
    };
    load(stage0, 0);
    for (int k = 0; k < p.pitch; k += 2 * kStep) {
        wait();
        if (k + kStep < p.pitch) load(stage1, k + kStep);
        multiply(stage0);
        wait();
        if (k + 2 * kStep < p.pitch) load(stage0, k + 2 * kStep);
        if (k + kStep < p.pitch) multiply(stage1);
    }
    // channels are the rows of a product: a lane has one token and four consecutive channels in each of four places
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = n0 + wn - BM + j * 32 + 8 * q + 4 * half;
            if (n >= p.N) continue;
            float scale[4], bias[4];
            channel_terms(p, n, scale, bias);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const size_t m = m0 + wm + i * 32 + r;
                if (m >= p.M) continue;
                const float sa = p.a_scale[m];
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)acc[i][j][4 * q + e] * sa * scale[e] + bias[e];
                put4<T>(p, m, n, v);
            }
        }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------
template <typename T> static hipError_t product(const ProductI8 &in, hipStream_t s, const char **name) {
    ProductArgs p{in.a, in.w, in.a_scale, in.w_scale, in.bias, in.out, in.M, in.ldo, in.N, rows8_pitch(in.K), 0, 0};
    const auto tiles = [&](int bm, int bn) {
        p.mtiles = (unsigned)((in.M + bm - 1) / bm);
        p.ntiles = (in.N + bn - 1) / bn;
        return (unsigned long long)p.mtiles * p.ntiles;
    };
    if (tiles(128, 128) >= 256) {
        if (tiles(256, 256) >= 256) {
            *name = "product8_tile<256,256>";
            hipLaunchKernelGGL((product8_tile_kernel<T, 2, 4, 4, 2>), dim3((unsigned)tiles(256, 256)), dim3(512), 0, s, p);
        } else {
            *name = "product8_tile<128,128>";
            hipLaunchKernelGGL((product8_tile_kernel<T, 2, 2, 2, 2>), dim3((unsigned)tiles(128, 128)), dim3(256), 0, s, p);
        }
    } else if (in.M <= 16) {
        *name = "product8_small<1,1>";
        hipLaunchKernelGGL((product8_small_kernel<T, 1, 1, 8>), dim3((unsigned)tiles(16, 16)), dim3(512), 0, s, p);
    } else {
        *name = "product8_small<2,2>";
        hipLaunchKernelGGL((product8_small_kernel<T, 2, 2, 4>), dim3((unsigned)tiles(32, 32)), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

hipError_t launch_matmul_i8(const ProductI8 &p, hipStream_t s, const char **name) {
    return p.out_dtype == GSPC_F32 ? product<float>(p, s, name) : product<uint16_t>(p, s, name);
}

}  // namespace gspc
