// out[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k] + bias[n], a and w 8-bit rows: integer sums on the matrix cores, exact.
#include "product_common.h"
#include "tokens_internal.h"

namespace gspc {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct ProductArgs {
    const int8_t *a, *w;
    const float *a_scale, *w_scale, *bias;
    void *out;
    size_t M, ldo;
    int N, pitch;
    unsigned mtiles, ntiles;
    int past;               // out is stored past the caches
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
// A block has 16 TN channels x 16 TM tokens; its waves split the reduction into stretches, operands straight from memory into the
// registers of v_mfma_i32_16x16x64_i8 (channels are the rows, tokens the columns of its result), DEEP steps of 64 in flight, and join
// their sums in LDS.  One token x 4096 x 4096: 5.0 us with its launch (16.8 MB), 8192 x 8192 12.8 us, 5.2 TB/s.
template <typename T, int TN, int TM, int WAVES, int DEEP>
__global__ __launch_bounds__(64 * WAVES) void product8_small_kernel(ProductArgs p) {
    __shared__ i32x4 s_part[WAVES][TN * TM][kWave];
    const unsigned nt = blockIdx.x % p.ntiles, mt = blockIdx.x / p.ntiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n0 = nt * 16 * TN;
    const size_t m0 = (size_t)mt * 16 * TM;
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const unsigned row = lane % 16, col = lane / 16 * 16, lane_off = row * p.pitch + col;
    const int steps = (p.pitch + 63) / 64, share = (steps + WAVES - 1) / WAVES;
    const int first = wave * share, last = min(first + share, steps);
    i32x4 acc[TN][TM] = {}, w[DEEP][TN], a[DEEP][TM];
    const auto load = [&](int d, int step) {        // (out of range past the row's end)
        const int k = step * 64;
        const unsigned off = k + (int)col < p.pitch ? lane_off + k : kOob;
#pragma unroll
        for (int i = 0; i < TN; ++i)
            w[d][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off == kOob ? kOob : off + i * 16 * p.pitch, 0, 0));
#pragma unroll
        for (int j = 0; j < TM; ++j)
            a[d][j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, off == kOob ? kOob : off + j * 16 * p.pitch, 0, 0));
    };
    const auto multiply = [&](int d) {
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[d][i], a[d][j], acc[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int d = 0; d < DEEP; ++d)
        if (first + d < last) load(d, first + d);
    for (int step = first; step < last; step += DEEP) {
#pragma unroll
        for (int d = 0; d < DEEP; ++d)
            if (step + d < last) {
                multiply(d);
                if (step + d + DEEP < last) load(d, step + d + DEEP);
            }
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) s_part[wave][i * TM + j][lane] = acc[i][j];
    // (the scales travel while the waves wait for one another)
    const auto terms = [&](int t, float (&scale)[4], float (&bias)[4], float &sa, size_t &m, int &n) {
        const int tile = t / kWave, l = t % kWave;
        m = m0 + tile % TM * 16 + l % 16;
        n = n0 + tile / TM * 16 + l / 16 * 4;
        channel_terms(p, n, scale, bias);
        sa = p.a_scale[m < p.M ? m : p.M - 1];
    };
    constexpr int EACH = (TN * TM + WAVES - 1) / WAVES;
    float scale[EACH][4], bias[EACH][4], sa[EACH];
    size_t m[EACH];
    int n[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if ((e * WAVES + wave) < TN * TM) terms(e * 64 * WAVES + threadIdx.x, scale[e], bias[e], sa[e], m[e], n[e]);
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int tile = e * WAVES + wave;
        if (tile >= TN * TM) break;
        i32x4 sum = s_part[0][tile][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += s_part[v][tile][lane];
        if (m[e] < p.M && n[e] < p.N) {
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = (float)sum[c] * sa[e] * scale[e][c] + bias[e][c];
            put4<T>(p, m[e], n[e], v);
        }
    }
}

// ---- many tokens: tiles through LDS ---------------------------------------------------------------------------------------------
constexpr int kStep = 128;              // bytes of a row that one stage holds: a cache line (stages of 64 bytes, twice as many of
                                        // them, make two requests of a line: 8192 x 4096 x 8192 took 285 us)

// WM x WN waves of TM x TN products 32x32x32 each.  STAGES stages hold 128 bytes of BM + BN rows each, brought by loads that write
// LDS directly (16 bytes a lane, eight rows a wave), STAGES - 1 ahead of the products.  Within a row the 16-byte pieces are permuted by the row's number, so that the
// lanes that read one column of pieces spread over all banks; a load's lanes fetch from the addresses that this asks for.
// 8192 x 4096 x 8192 to bf16: 217 to 239 us, 2.3 to 2.5 POP/s.  A copy of the loop without its loads took 210, and whole products of zeros a
// quarter less than of random values: the chip's power sets the clock.  12544 x 1024 x 512 (196 tiles, one round): 12.9 us.  Stages of
// 64 bytes, four of them, took 285 us instead of 255 (two requests for a cache line).  Four waves of 128 x 128 products each instead of eight
// of 128 x 64 were level where K is long and behind where it is short.
template <typename T, int WM, int WN, int TM, int TN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void product8_tile_kernel(ProductArgs p) {
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, ROWS = BM + BN, LOADS = ROWS / 8 / WAVES;
    constexpr int STAGE = ROWS * kStep;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "a load is of one operand");
    __shared__ __attribute__((aligned(16))) char stages[STAGES * STAGE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const uint2 tile = tile_of(p.mtiles, p.ntiles, blockIdx.x);
    const size_t m0 = (size_t)tile.x * BM;
    const int n0 = tile.y * BN;
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const auto swizzle = [](int row) { return (row & 7) ^ (row >> 3 & 1); };

    // Load i of this wave: rows base .. base + 7; lane l has the piece that belongs into its place of row base + l / 8.
    const int piece[2] = {(lane & 7) ^ swizzle(lane >> 3), (lane & 7) ^ swizzle(8 + (lane >> 3))};
    const unsigned lane_off = (unsigned)(lane / 8) * p.pitch;
    const auto load_one = [&](unsigned stage, int k, int i) {
        const bool tokens = i < BM / (8 * WAVES);
        const int base = (i * WAVES + wave) * 8, at = k + piece[wave & 1] * 16;     // (WAVES is even)
        // (out of range past the row's end, from the lane's own offset on: no branch, which would make two loads of one)
        const unsigned past = at < p.pitch ? 0u : kOob;
        const unsigned off = (lane_off + at + (unsigned)(base - (tokens ? 0 : BM)) * p.pitch) | past;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(tokens ? ra : rw, (__attribute__((address_space(3))) void *)(stages + stage + base * kStep), 16,
                                                 off, 0, 0, 0);
    };
    i32x16 acc[TM][TN] = {};
    const int wm = wave / WN * TM * 32, wn = wave % WN * TN * 32, r = lane % 32, half = lane / 32;
    constexpr int PARTS = kStep / 32, READS = TM + TN;
    i32x4 op[2][READS];                             // operands of this part of a stage, and of the next: tokens, channels
    const auto read_one = [&](unsigned stage, int k, int i) {
        const int row = i < TM ? wm + i * 32 : BM + wn + (i - TM) * 32;
        return *reinterpret_cast<const i32x4 *>(stages + stage + (row + r) * kStep + ((2 * k + half) ^ swizzle(r)) * 16);
    };

    constexpr int SCALES = ((BM > BN ? BM : BN) + 64 * WAVES - 1) / (64 * WAVES);
    float w_scale[SCALES], bias[SCALES], a_scale[SCALES];
#pragma unroll
    for (int i = 0; i < SCALES; ++i) {
        const int t = i * 64 * WAVES + threadIdx.x, n = min(n0 + t, p.N - 1);
        const size_t m = m0 + t < p.M ? m0 + t : p.M - 1;
        w_scale[i] = p.w_scale[n];
        bias[i] = p.bias ? p.bias[n] : 0.f;
        a_scale[i] = p.a_scale[m];
    }
    // A stage in parts of 32 bytes of a row.  While a part is multiplied the next part's operands are read, channels first: a part
    // begins with one token's products.  Before the next stage's are read that has to be there, and every wave has all of this one
    // in registers: what comes STAGES later is loaded into its place, FIRST loads there and the others behind the next stage's
    // first products, as evenly as products allow: a wave that waits for the memory path to take its load multiplies nothing.
    // (That wait stands behind the last part's first products, not before.)
    constexpr int SLOTS = READS, SKIP = READS / 4, FIRST = (LOADS + 1) / 2;
    const auto share = [](int all, int slots, int t) { return all * t / slots; };     // of `all`, those before slot t of `slots`
#pragma unroll
    for (int t = 0; t < STAGES; ++t)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (t + 1 < STAGES || i < FIRST) load_one(t * STAGE, t * kStep, i);
            __builtin_amdgcn_sched_barrier(0);      // loads are counted: in this order
        }
    wait_loads<(STAGES - 2) * LOADS + FIRST>();
    barrier_of_block();
#pragma unroll
    for (int t = 0; t < READS; ++t) op[0][t] = read_one(0, 0, t);
    unsigned stage = 0, before = (STAGES - 1) * STAGE;      // of step k, and of the one before, where k + STAGES - 1 comes
    for (int k = 0; k < p.pitch; k += kStep) {
        const unsigned next = stage + STAGE == STAGES * STAGE ? 0 : stage + STAGE;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            const bool last = q == PARTS - 1;
#pragma unroll
            for (int t = 0; t < SLOTS; ++t) {
                if (last && t == SKIP) {
                    wait_loads<(STAGES - 2) * LOADS>();
                    barrier_of_block();
                    __builtin_amdgcn_sched_barrier(0);
                }
                const int s = last ? t - SKIP : t, slots = last ? SLOTS - SKIP : SLOTS;
                if (s >= 0) {
#pragma unroll
                    for (int u = share(READS, slots, s); u < share(READS, slots, s + 1); ++u) {
                        const int o = u < TN ? TM + u : u - TN;
                        op[(q + 1) & 1][o] = last ? read_one(next, 0, o) : read_one(stage, q + 1, o);
                    }
                    if (q == 0)
#pragma unroll
                        for (int u = share(LOADS - FIRST, slots, s); u < share(LOADS - FIRST, slots, s + 1); ++u)
                            load_one(before, k + (STAGES - 1) * kStep, FIRST + u);
                    if (last)
#pragma unroll
                        for (int u = share(FIRST, slots, s); u < share(FIRST, slots, s + 1); ++u) load_one(stage, k + STAGES * kStep, u);
                }
#pragma unroll
                for (int c = share(TM * TN, SLOTS, t); c < share(TM * TN, SLOTS, t + 1); ++c)
                    acc[c / TN][c % TN] =
                        __builtin_amdgcn_mfma_i32_32x32x32_i8(op[q & 1][TM + c % TN], op[q & 1][c / TN], acc[c / TN][c % TN], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        before = stage;
        stage = next;
    }
    __builtin_amdgcn_s_waitcnt(0);                  // (loads of zeros past the end)
    // Channels are the rows of a product: a lane has one token and four consecutive channels in each of four places.  Each wave
    // turns its own 32 tokens at a time through LDS (in the stages' place, which nobody reads any more), so that a store writes whole
    // lines of a token; so do the scales, loaded before the products.
    constexpr int WAVE_N = TN * 32, PITCH = WAVE_N * sizeof(T) + 16, LANES = WAVE_N * sizeof(T) / 16, EACH = 16 / sizeof(T);
    static_assert(WAVES * 32 * PITCH + 4 * (2 * BN + BM) <= STAGES * STAGE, "fits the stages");
    __syncthreads();
    float *s_scale = reinterpret_cast<float *>(stages), *s_bias = s_scale + BN, *s_token = s_bias + BN;
#pragma unroll
    for (int i = 0; i < SCALES; ++i) {
        const int t = i * 64 * WAVES + threadIdx.x;
        if (t < BN) s_scale[t] = w_scale[i], s_bias[t] = bias[i];
        if (t < BM) s_token[t] = a_scale[i];
    }
    __syncthreads();
    char *turn = stages + 4 * (2 * BN + BM) + wave * 32 * PITCH;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const float sa = s_token[wm + i * 32 + r];
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = j * 32 + 8 * q + 4 * half;
                const f32x4 sw = *reinterpret_cast<const f32x4 *>(s_scale + wn + n), sb = *reinterpret_cast<const f32x4 *>(s_bias + wn + n);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)acc[i][j][4 * q + e] * sa * sw[e] + sb[e];
                if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(turn + r * PITCH + n * 4) = (f32x4){v[0], v[1], v[2], v[3]};
                else *reinterpret_cast<u32x2 *>(turn + r * PITCH + n * 2) = (u32x2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
            }
        barrier_of_wave();            // (LDS operations of one wave are in order)
#pragma unroll
        for (int t = 0; t < 32; t += kWave / LANES) {
            const int row = t + lane / LANES, n = lane % LANES * EACH;
            const size_t m = m0 + wm + i * 32 + row;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(turn + row * PITCH + lane % LANES * 16);
            if (m < p.M) {
                T *o = static_cast<T *>(p.out) + m * p.ldo + n0 + wn + n;
                const int left = p.N - n0 - wn - n;
                if (left >= EACH) store_vector(reinterpret_cast<u32x4_any *>(o), v, p.past);
                else {
#pragma unroll
                    for (int e = 0; e < EACH; ++e)
                        if (e < left) {
                            if constexpr (sizeof(T) == 4) o[e] = __uint_as_float(v[e]);
                            else o[e] = (uint16_t)(v[e / 2] >> (e % 2 * 16));
                        }
                }
            }
        }
        barrier_of_wave();
    }
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------
template <typename T> static hipError_t product(const ProductI8 &in, hipStream_t s, const char **name) {
    const unsigned pitch = rows8_pitch(in.K);
    const auto count = [](size_t all, unsigned of) { return (unsigned)((all - 1) / of + 1); };
    const auto tiles = [&](int bm, int bn) { return (unsigned long long)count(in.M, bm) * count(in.N, bn); };
    // Past the caches (M x K x N, us through them and past): 8192 x 4096 x 8192, 255 and 240; 16384 x 256 x 1024, 12.1 and 10.2.  From 16 MB on only
    // rows of whole pieces: 16384 x 256 x 1001, 13.6 and 17.3, 100000 x 64 x 1001 55.8 and 109 (below, 8582 x 64 x 501 7.1 and 7.8, 11976 x 1024 x
    // 501 14.4 and 13.5).
    const size_t bytes = in.M * in.N * sizeof(T);
    const int past = bytes >= kPastCaches && (bytes < 2 * kPastCaches || whole_pieces(in.out, in.N * sizeof(T), in.ldo * sizeof(T)));
    const auto run = [&](auto kern, unsigned bm, unsigned bn, unsigned threads, const char *name_of) {
        *name = name_of;
        const unsigned most = most_blocks(threads), nt = count(in.N, bn) < most ? count(in.N, bn) : most;
        const size_t m_step = (size_t)(most / nt) * bm, n_step = (size_t)nt * bn;       // of one launch at most
        for (size_t m = 0; m < in.M; m += m_step)
            for (size_t n = 0; n < (size_t)in.N; n += n_step) {
                const size_t rows = in.M - m < m_step ? in.M - m : m_step, cols = in.N - n < n_step ? in.N - n : n_step;
                const ProductArgs p{in.a + m * pitch, in.w + n * pitch, in.a_scale + m, in.w_scale + n, in.bias ? in.bias + n : nullptr,
                                    static_cast<T *>(in.out) + m * in.ldo + n, rows, in.ldo, (int)cols, (int)pitch, count(rows, bm), count(cols, bn),
                                    past};
                hipLaunchKernelGGL(kern, dim3(p.mtiles * p.ntiles), dim3(threads), 0, s, p);
            }
    };
    // The largest tile that is more than half full and still gives most compute units one (M x K x N, us; both sides):
    //   256 x 256 from 160 tiles on: 12544 x 512 x 1024 has 196, 15.0 against 17.1 in tiles of 128; 2048 x 2048 x 4096 has 128, 27.8
    //   against 22.4.  Not for 128 tokens or filters and fewer: 128 x 4096 x 50257, 44.4 against 34.0 in tiles of 128 (129 tokens 43.7
    //   against 53); 50000 x 512 x 128, 12.3 against 7.9 (129 filters 13.4 against 14.7);
    //   128 x 128 from 256 tiles on: 2048 x 2048 x 4096 has 512, 22.4 against 29 in 64 x 128; 512 x 4096 x 4096 has 128, 18.3 against 15.8.
    //   Not for 64 tokens and fewer: 64 x 4096 x 32768, 25.3 against 22.1 in 64 x 128 (96 tokens 25.8 against 24.2, 128 x 4096 x 50257 34.0
    //   against 44);
    //   64 x 128 where 32 x 32 without staging would be more than one block for each compute unit: 512 x 4096 x 4096, 15.8 against
    //   59; 200 x 1024 x 1024 (224 blocks without staging), 5.9 against 4.4.
    //   or where its steps are few: 133 x 195 x 3608, 3.7 without staging, 4.4 in 64 x 128.
    // Up to 16 tokens: 1 x 4096 x 4096, 5.1 in blocks of 16 channels, 7.2 in blocks of 32 x 32; unless tiles of 64 x 128 give every compute
    // unit one: 16 x 4096 x 32768, 30.9 against 21.0 (1 token 24.8 against 20.4; 1 x 4096 x 16384 has 128 tiles, 13.8 against 12.9).
    if (in.M > 128 && in.N > 128 && tiles(256, 256) >= 160) run(product8_tile_kernel<T, 2, 4, 4, 2, 2>, 256, 256, 512, "product8_tile<256,256>");
    else if (in.M > 64 && tiles(128, 128) >= 256) run(product8_tile_kernel<T, 2, 2, 2, 2, 2>, 128, 128, 256, "product8_tile<128,128>");
    else if (in.M <= 16 && tiles(64, 128) < 256) run(product8_small_kernel<T, 1, 1, 8, 4>, 16, 16, 512, "product8_small<1,1>");
    else if (tiles(32, 32) <= 256 || tiles(32, 32) * ((pitch + 63) / 64) <= 2560) run(product8_small_kernel<T, 2, 2, 8, 2>, 32, 32, 512, "product8_small<2,2>");
    else run(product8_tile_kernel<T, 2, 2, 1, 2, 3>, 64, 128, 256, "product8_tile<64,128>");
    return hipGetLastError();
}

hipError_t launch_matmul_i8(const ProductI8 &p, hipStream_t s, const char **name) {
    return p.out_dtype == GSPC_F32 ? product<float>(p, s, name) : product<uint16_t>(p, s, name);
}

}  // namespace gspc
