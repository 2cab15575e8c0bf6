// out[m][n] = sum over blocks j of 128 of 2^(a_scale[m][j] + w_scale[n][j]) sum_k a[m][k] w[n][k], + bias[n]: a and w 8-bit float rows.
//
// For bf16 outputs the matrix cores take the powers of two with the operands (v_mfma_scale_f32_*_f8f6f4, a byte for each lane's row), so that the sum
// over all blocks stays in their fp32 accumulators and scaling costs no instruction.  These instructions add eight products at a time with no bit below
// 2^-13 of the largest one's exponent (in e4m3 all do, the scaled ones and the older ones alike), each cut off there: less than 2^-10 of sum |a w|, and
// 1.5e-5 of the result on random values, a hundredth of its rounding to bf16.  For fp32 outputs that is too much.  There the operands are widened to bf16
// with their power of two (exact: four significant bits, in steps of 2^-133 and below 2^128) and multiplied by the bf16 instructions, whose sums keep 24 bits
// (5e-9 on random values); the
// peak is half of that (loops in registers: 3.7 PFLOP/s and, with the widening, 1.46).
#include "float8.h"
#include "product_common.h"
#include "tokens_internal.h"

namespace gspc {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct ProductF8Args {
    const uint8_t *a, *a_scale, *w, *w_scale;
    const float *bias;
    void *out;
    size_t M, ldo;
    size_t part;            // elements between the outputs of two stretches of K
    int N, pitch, s_pitch;
    int stretch;            // steps of 128 columns of a stretch of K, and
    unsigned tiles;         // blocks of one
    unsigned mtiles, ntiles;
    int past;               // out is stored past the caches
};

__device__ __forceinline__ i32x8 both(u32x4 lo, u32x4 hi) {
    return (i32x8){(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// Eight columns as bf16, times 2^(code - 127).
__device__ __forceinline__ bf16x8 widened(int lo, int hi, float down) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, down, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, down, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, down, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, down, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// A lane's 32 columns of one row.
struct Wide {
    bf16x8 part[4];
};
__device__ __forceinline__ Wide widened(const i32x8 &v, unsigned code) {
    const float down = block_down(code & 255);
    Wide w;
#pragma unroll
    for (int s = 0; s < 4; ++s) w.part[s] = widened(v[2 * s], v[2 * s + 1], down);
    return w;
}

// ---- few tokens or few outputs: no staging --------------------------------------------------------------------------------------
// A block has 16 TN channels x 16 TM tokens; its waves split the reduction into stretches, operands straight from memory into the registers of
// v_mfma_scale_f32_16x16x128 (channels are the rows, tokens the columns of its result; a lane's 32 columns are two pieces of 16, so that a
// load of sixteen rows is of 64 bytes of each), DEEP steps of 128 in flight, and join their sums in LDS.
// Bound by latency: 1 x 4096 x 4096, 17 MB, 6.0 us and 5.8 for the call; 1 x 4096 x 50257, 206 MB, 43 us (4.8 TB/s).  WIDE: operands as bf16.
template <typename T, bool WIDE, int TN, int TM, int WAVES, int DEEP>
__global__ __launch_bounds__(64 * WAVES) void product_f8_small_kernel(ProductF8Args p) {
    __shared__ f32x4 s_part[WAVES][TN * TM][kWave];
    const unsigned part = blockIdx.x / p.tiles, tile = blockIdx.x - part * p.tiles, nt = tile % p.ntiles, mt = tile / p.ntiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n0 = nt * 16 * TN;
    const size_t m0 = (size_t)mt * 16 * TM;
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const __amdgpu_buffer_rsrc_t rsw = bytes_at(p.w_scale + (size_t)n0 * p.s_pitch, (size_t)(p.N - n0) * p.s_pitch);
    const __amdgpu_buffer_rsrc_t rsa = bytes_at(p.a_scale + m0 * p.s_pitch, (p.M - m0) * p.s_pitch);
    const unsigned row = lane % 16, lane_off = row * p.pitch + lane / 16 * 16, lane_scale = row * p.s_pitch;
    const int begin = (int)part * p.stretch, end = min(begin + p.stretch, p.pitch / kBlock8), share = (end - begin + WAVES - 1) / WAVES;
    const int first = begin + wave * share, last = min(first + share, end);
    static_assert(TN * TM <= WAVES, "a wave joins one product at most");
    float bias[4] = {};                             // (on its way with the operands, not behind them)
    if (p.bias && wave < TN * TM)
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[e] = p.bias[min(n0 + wave / TM * 16 + lane / 16 * 4 + e, p.N - 1)];
    f32x4 acc[TN][TM] = {};
    u32x4 w[DEEP][TN][2], a[DEEP][TM][2];
    static_assert(DEEP <= 4, "DEEP steps' bytes are in two words");
    uint64_t sw[TN], sa[TM], next_sw[TN], next_sa[TM];
    const auto load_scales = [&](int step) {        // of this and the next DEEP - 1 steps, whatever their place in their words
        const unsigned s = step & ~3;
#pragma unroll
        for (int i = 0; i < TN; ++i) next_sw[i] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(rsw, lane_scale + i * 16 * p.s_pitch + s, 0, 0));
#pragma unroll
        for (int j = 0; j < TM; ++j) next_sa[j] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(rsa, lane_scale + j * 16 * p.s_pitch + s, 0, 0));
    };
    const auto load = [&](int d, int step) {
        const unsigned k = step * kBlock8;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            const unsigned off = lane_off + i * 16 * p.pitch + k;
            w[d][i][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off, 0, 0));
            w[d][i][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off + 64, 0, 0));
        }
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            const unsigned off = lane_off + j * 16 * p.pitch + k;
            a[d][j][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, off, 0, 0));
            a[d][j][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, off + 64, 0, 0));
        }
    };
    const auto multiply = [&](int d, int step) {
        const int turn = ((step & 3) + d) * 8;
        if constexpr (WIDE) {
            Wide ww[TN];
#pragma unroll
            for (int i = 0; i < TN; ++i) ww[i] = widened(both(w[d][i][0], w[d][i][1]), (unsigned)(sw[i] >> turn));
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const Wide aw = widened(both(a[d][j][0], a[d][j][1]), (unsigned)(sa[j] >> turn));
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int s = 0; s < 4; ++s) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ww[i].part[s], aw.part[s], acc[i][j], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(both(w[d][i][0], w[d][i][1]), both(a[d][j][0], a[d][j][1]), acc[i][j], 0,
                                                                                  0, 0, (int)(sw[i] >> turn), 0, (int)((unsigned)(sa[j] >> turn)));
        }
    };
    load_scales(first);
#pragma unroll
    for (int d = 0; d < DEEP; ++d)
        if (first + d < last) load(d, first + d);
    for (int step = first; step < last; step += DEEP) {
#pragma unroll
        for (int i = 0; i < TN; ++i) sw[i] = next_sw[i];
#pragma unroll
        for (int j = 0; j < TM; ++j) sa[j] = next_sa[j];
        if (step + DEEP < last) load_scales(step + DEEP);
#pragma unroll
        for (int d = 0; d < DEEP; ++d)
            if (step + d < last) {
                multiply(d, step);
                if (step + d + DEEP < last) load(d, step + d + DEEP);
            }
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j) s_part[wave][i * TM + j][lane] = acc[i][j];
    __syncthreads();
    if (wave >= TN * TM) return;
    f32x4 sum = s_part[0][wave][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum += s_part[v][wave][lane];
    const size_t m = m0 + wave % TM * 16 + row;
    const int n = n0 + wave / TM * 16 + lane / 16 * 4;
    if (m >= p.M || n >= p.N) return;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = sum[e] + bias[e];
    T *o = static_cast<T *>(p.out) + part * p.part + m * p.ldo + n;
    if (n + 3 < p.N) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_any *>(o) = (f32x4){v[0], v[1], v[2], v[3]};
        else *reinterpret_cast<u32x2_any *>(o) = (u32x2){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (n + e < p.N) put(o + e, v[e]);
    }
}

// ---- many tokens: tiles through LDS ---------------------------------------------------------------------------------------------
// WM x WN waves of TM x TN products 32x32x64 each.  STAGES stages hold 128 columns (a block, a cache line) of BM + BN rows each, brought by loads
// that write LDS directly (16 bytes a lane, eight rows a wave), STAGES - 1 ahead of the products; the powers of two of four blocks are a
// word of a row and come the same way, once in four stages.  Within a row the 16-byte pieces are permuted by the row's number, so that the lanes that read
// one column of pieces spread over all banks; a load's lanes fetch from the addresses that this asks for.  A lane's 32 columns of a product are two
// such pieces; which columns of the block they are does not matter as long as both operands agree.
//
// Bound by the matrix instructions where there is enough work: 8192 x 4096 x 8192 to bf16 in 256 x 256 takes 219 us (2.5 PFLOP/s; the
// library's product without scales 216).  WIDE: each wave widens all of its operands, four clocks for 128 values (loops in registers, two waves a SIMD:
// 32 such instructions 58 ns, exclusive ors 37; with 8 products that do not wait for them 160, where these alone take 147: they go side by side).  A step
// of 64 x 64 in a wave (128 x 128) has 512 clocks of them and 1024 of products, and these bound it (8192 x 4096 x 8192 to fp32: 461 us, 1.19 PFLOP/s); one of 32 x 32
// (64 x 128) 256 of either, and with loads and a barrier a step neither bounds it (1024 x 12544 x 512 in four stretches, 23.9 us and a join of 4.8: matrix
// instructions at work 29 % of the time, vector instructions half of it; a wave waits 37 % of its time for loads and its block, 25 % for its turn).
template <typename T, bool WIDE, int WM, int WN, int TM, int TN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void product_f8_tile_kernel(ProductF8Args p) {
    constexpr int WAVES = WM * WN, BM = 32 * WM * TM, BN = 32 * WN * TN, ROWS = BM + BN, LOADS = ROWS / 8 / WAVES;
    constexpr int STAGE = ROWS * kBlock8;
    static_assert(BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "a load is of one operand");
    static_assert(BM % kWave == 0 && BN % kWave == 0 && ROWS / kWave <= WAVES, "a wave loads the powers of 64 rows of one operand");
    // (one array: between reads of one and loads into another the compiler waits for all loads)
    constexpr int SCALES = STAGES * STAGE;
    __shared__ __attribute__((aligned(16))) char stages[SCALES + 2 * ROWS * 4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const unsigned part = blockIdx.x / p.tiles;
    const uint2 tile = tile_of(p.mtiles, p.ntiles, blockIdx.x - part * p.tiles);
    const size_t m0 = (size_t)tile.x * BM;
    const int n0 = tile.y * BN;
    const __amdgpu_buffer_rsrc_t ra = bytes_at(p.a + m0 * p.pitch, (p.M - m0) * p.pitch);
    const __amdgpu_buffer_rsrc_t rw = bytes_at(p.w + (size_t)n0 * p.pitch, (size_t)(p.N - n0) * p.pitch);
    const __amdgpu_buffer_rsrc_t rsa = bytes_at(p.a_scale + m0 * p.s_pitch, (p.M - m0) * p.s_pitch);
    const __amdgpu_buffer_rsrc_t rsw = bytes_at(p.w_scale + (size_t)n0 * p.s_pitch, (size_t)(p.N - n0) * p.s_pitch);
    const auto swizzle = [](int row) { return (row & 7) ^ (row >> 3 & 1); };
    const int begin = (int)part * p.stretch, end = min(begin + p.stretch, p.pitch / kBlock8);      // steps

    // Load i of this wave: rows base .. base + 7; lane l has the piece that belongs into its place of row base + l / 8.
    const int piece[2] = {(lane & 7) ^ swizzle(lane >> 3), (lane & 7) ^ swizzle(8 + (lane >> 3))};
    const unsigned lane_off = (unsigned)(lane / 8) * p.pitch;
    const auto load_one = [&](unsigned stage, int step, int i) {
        const bool tokens = i < BM / (8 * WAVES);
        const int base = (i * WAVES + wave) * 8, at = step * kBlock8 + piece[wave & 1] * 16;       // (WAVES is even)
        // (out of range past the stretch's end, from the lane's own offset on: no branch, which would make two loads of one)
        const unsigned past = step < end ? 0u : kOob;
        const unsigned off = (lane_off + at + (unsigned)(base - (tokens ? 0 : BM)) * p.pitch) | past;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(tokens ? ra : rw, (__attribute__((address_space(3))) void *)(stages + stage + base * kBlock8), 16,
                                                 off, 0, 0, 0);
    };
    const auto load_scales = [&](int step) {        // of steps step .. step + 3, step a multiple of four
        if (wave < ROWS / kWave) {
            const bool tokens = wave < BM / kWave;
            const unsigned at = (unsigned)(wave * kWave - (tokens ? 0 : BM) + lane) * p.s_pitch + step;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(tokens ? rsa : rsw, (__attribute__((address_space(3))) void *)(stages + SCALES + ((step / 4 & 1) * ROWS + wave * kWave) * 4), 4, step < end ? at : kOob, 0, 0, 0);
        }
    };
    f32x16 acc[TM][TN] = {};
    const int wm = wave / WN * TM * 32, wn = wave % WN * TN * 32, r = lane % 32, half = lane / 32;
    const auto read_one = [&](unsigned stage, int q, int row) {
        const char *at = stages + stage + (row + r) * kBlock8;
        return both(*reinterpret_cast<const u32x4 *>(at + ((2 * q + half) ^ swizzle(r)) * 16),
                    *reinterpret_cast<const u32x4 *>(at + ((2 * q + 4 + half) ^ swizzle(r)) * 16));
    };
    i32x8 a[TM], w[2][TN];                          // operands of this half of a stage; channels of the next one too
    unsigned sa[TM], sw[TN];
    const auto read_scales = [&](int step) {        // (the products take the word's low byte)
        const int turn = (step & 3) * 8;
        const unsigned *at = reinterpret_cast<const unsigned *>(stages + SCALES) + (step >> 2 & 1) * ROWS + r;
#pragma unroll
        for (int i = 0; i < TM; ++i) sa[i] = at[wm + i * 32] >> turn;
#pragma unroll
        for (int j = 0; j < TN; ++j) sw[j] = at[BM + wn + j * 32] >> turn;
    };
    Wide ww[WIDE ? TN : 1];
    const auto multiply = [&](int q, int i) {
        if constexpr (WIDE) {
            if (i == 0)
#pragma unroll
                for (int j = 0; j < TN; ++j) ww[j] = widened(w[q][j], sw[j]);
            const Wide aw = widened(a[i], sa[i]);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ww[j].part[s], aw.part[s], acc[i][j], 0, 0, 0);
            return;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[q][j], a[i], acc[i][j], 0, 0, 0, (int)sw[j], 0, (int)sa[i]);
    };

    // A stage in two halves of its columns.  As soon as a token fragment's products are under way the next half's is read into its registers.
    // Before the next stage's are read that has to be there, and every wave has all of this one in registers: what comes STAGES
    // later is loaded into its place, a few loads behind each fragment's products.  (That wait stands behind the last half's first products.)
    load_scales(begin & ~3);
    if (begin & 3) load_scales((begin & ~3) + 4);       // (a stretch may begin anywhere)
#pragma unroll
    for (int t = 0; t < STAGES; ++t)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            load_one(t * STAGE, begin + t, i);
            __builtin_amdgcn_sched_barrier(0);      // loads are counted: in this order
        }
    wait_loads<(STAGES - 1) * LOADS>();
    barrier_of_block();
#pragma unroll
    for (int j = 0; j < TN; ++j) w[0][j] = read_one(0, 0, BM + wn + j * 32);
#pragma unroll
    for (int i = 0; i < TM; ++i) a[i] = read_one(0, 0, wm + i * 32);
    read_scales(begin);
    unsigned stage = 0;
    for (int step = begin; step < end; ++step) {
        const unsigned next = stage + STAGE == STAGES * STAGE ? 0 : stage + STAGE;
        if ((step & 3) == 0) load_scales(step + 4);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            multiply(0, i);
            if (i < TN) w[1][i] = read_one(stage, 1, BM + wn + i * 32);
            if (i == TM - 1)
#pragma unroll
                for (int j = TM; j < TN; ++j) w[1][j] = read_one(stage, 1, BM + wn + j * 32);
            a[i] = read_one(stage, 1, wm + i * 32);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            multiply(1, i);
            if (i == 0) {
                __builtin_amdgcn_sched_barrier(0);
                wait_loads<(STAGES - 2) * LOADS>();
                barrier_of_block();
                __builtin_amdgcn_sched_barrier(0);
            }
            if (i < TN) w[0][i] = read_one(next, 0, BM + wn + i * 32);
            if (i == TM - 1)
#pragma unroll
                for (int j = TM; j < TN; ++j) w[0][j] = read_one(next, 0, BM + wn + j * 32);
            a[i] = read_one(next, 0, wm + i * 32);
#pragma unroll
            for (int u = LOADS * i / TM; u < LOADS * (i + 1) / TM; ++u) load_one(stage, step + STAGES, u);
            __builtin_amdgcn_sched_barrier(0);
        }
        read_scales(step + 1);                      // (no branch here: the products would be moved behind it, all of them)
        stage = next;
    }
    __builtin_amdgcn_s_waitcnt(0);                  // (loads of zeros past the end)
    // Channels are the rows of a product: a lane has one token and four consecutive channels in each of four places.  Each wave
    // turns its own 32 tokens at a time through LDS (in the stages' place, which nobody reads any more), so that a store writes whole
    // lines of a token.
    constexpr int WAVE_N = TN * 32, PITCH = WAVE_N * sizeof(T) + 16, LANES = WAVE_N * sizeof(T) / 16, EACH = 16 / sizeof(T);
    static_assert(WAVES * 32 * PITCH + 4 * BN <= STAGES * STAGE, "fits the stages");
    __syncthreads();
    float *s_bias = reinterpret_cast<float *>(stages);
    for (int t = threadIdx.x; t < BN; t += 64 * WAVES) s_bias[t] = p.bias ? p.bias[min(n0 + t, p.N - 1)] : 0.f;
    __syncthreads();
    char *turn = stages + 4 * BN + wave * 32 * PITCH;
    T *out = static_cast<T *>(p.out) + part * p.part;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = j * 32 + 8 * q + 4 * half;
                const f32x4 sb = *reinterpret_cast<const f32x4 *>(s_bias + wn + n);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e] + sb[e];
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
                T *o = out + m * p.ldo + n0 + wn + n;
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

// Sums of stretches of K, in their order (four of 1024 x 512: 4 us, latency).
template <typename T>
__global__ __launch_bounds__(256) void product_f8_join_kernel(const float *__restrict__ part, size_t each, unsigned parts, unsigned vectors, int N,
                                                              unsigned nv, unsigned m_nv, const float *__restrict__ bias, T *__restrict__ out, size_t ldo) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i >= vectors) return;
    const unsigned m = fast_div_any(i, nv, m_nv);
    const int n = (i - m * nv) * 4, some = min(4, N - n);
    const float *p = part + (size_t)m * N + n;
    float v[4] = {};
    if (some == 4) {
        for (unsigned k = 0; k < parts; k += 4) {       // four on their way at once, whether they are there or not (no branch in front of a load)
            f32x4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const f32x4_any *>(p + min(k + i, parts - 1) * each);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += k + i < parts ? x[i][e] : 0.f;
        }
    } else {
        for (unsigned k = 0; k < parts; ++k, p += each)
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < some) v[e] += p[e];
    }
    T *o = out + m * ldo + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < some) put(o + e, bias ? v[e] + bias[n + e] : v[e]);
}

// ---- launches ---------------------------------------------------------------------------------------------------------------------
enum { kSmall1, kSmall2, kTile64, kTile128, kTile256, kTile128Deep };
struct PlanF8 {
    int kernel, bm, bn, threads;
    int parts, stretch;     // stretches of K, and steps of each
};

static PlanF8 plan_f8(size_t M, int N, int K, bool wide) {
    const int steps = f8_pitch(K) / kBlock8;
    const auto tiles = [&](int bm, int bn) { return ((M + bm - 1) / bm) * (size_t)((N + bn - 1) / bn); };
    PlanF8 p;
    // (M x K x N, us of a call among others, bf16 outputs unless said; both sides)
    //   256 x 256 from 160 tiles on: 12544 x 512 x 1024 has 196, 13.0 against 15.8 in tiles of 128; 2048 x 512 x 4096 has 128, 12.0 against 9.0.  Not
    //   for 128 tokens or filters and fewer, where more than half of a tile is empty;
    //   128 x 128 from 192 tiles on: 1000 x 2000 x 3000 has 192, 11.9 against 13.0 in 64 x 128; 512 x 4096 x 4096 has 128, 17.3 against 16.3.  Four
    //   stages and eight waves where a compute unit has one block: 1000 x 2000 x 3000, 11.9 against 13.7 with four waves and 15.2 with two stages, too;
    //   12544 x 512 x 1024 (784 tiles), 20.1, 23.8 and 15.4.  Eight waves in 64 x 128 too: 400 x 1280 x 1001, 6.8 against 7.3 with four;
    //   without staging, in 16 x 16: for up to 16 tokens and 16384 filters (8 x 8192 x 8192, 15.0 against 16.5 in 64 x 128 and stretches; 16 x 4096 x
    //   32768, 36.2 against 33.1), for up to 8 and rows of 4096 on (1 x 4096 x 50257, 39.6 against 43.6; 8 x 4096 x 50257, 45.4 against 48.0; 12,
    //   49.2 against 48.2; 1 x 1024 x 50257, 15.3 against 11.1), or up to 256 blocks of up to 32 steps (64 x 512 x 512, 2.6 against 3.2 in 32 x 32;
    //   256 x 1024 x 1024, 6.7 against 4.4), or up to 64 (96 x 16384 x 160 in four stretches, 10.0 against 13.7; 256 x 50176 x 128 has 128, 28.4
    //   against 20.2); and in 32 x 32 for up to 256 blocks of up to 32 steps (64 x 4096 x 4096, 10.4 against 12.5 in 64 x 128 and stretches; 64 x
    //   8192 x 2048, 18.8 against 13.4), or more of few steps (5000 x 64 x 64, 3.7 against 4.2; operands as bf16 are widened for fewer products in 64
    //   x 128, 256 x 2048 x 2048 to fp32, 11.8 against 13.2, to bf16 11.1 against 8.9).
    const size_t small = tiles(16, 16), middle = tiles(32, 32);
    if (!wide && M > 128 && N > 128 && tiles(256, 256) >= 160) p = {kTile256, 256, 256, 512, 1, steps};
    else if (M > 64 && tiles(128, 128) >= 192) p = {tiles(128, 128) <= 256 ? kTile128Deep : kTile128, 128, 128, tiles(128, 128) <= 256 ? 512 : 256, 1, steps};
    else if ((M <= 16 && tiles(64, 128) <= 128) || (M <= 8 && steps >= 32) || (small <= 256 && steps <= 32) || small <= 64) p = {kSmall1, 16, 16, 512, 1, steps};
    else if ((middle <= 256 && steps <= 32) || (middle <= 640 && steps <= 2) || (wide && middle <= 512 && steps <= 16)) p = {kSmall2, 32, 32, 512, 1, steps};
    else p = {kTile64, 64, 128, 512, 1, steps};
    // Few blocks of a long sum: stretches of K, of 8 steps at least (32, where the block's waves share them), until every compute unit has a block.  512 x
    // 12544 x 512 has 32 tiles: 36.2 whole, 14.3 in eight stretches and their join; 512 x 4096 x 4096 has 128, 15.6 and 22.7 in two.  Stretches of whole
    // words of powers of two (of 28 steps instead of 25) take 1 us more on 1024 x 12544 x 512 to fp32, of 27.
    const size_t count = tiles(p.bm, p.bn);
    if (count <= 64 && (p.kernel == kSmall1 || p.kernel == kTile64)) {
        const int want = (int)(256 / count), most = steps / (p.kernel == kSmall1 ? 32 : 8), parts = want < most ? want : most;
        if (parts > 1) {
            p.stretch = (steps + parts - 1) / parts;
            p.parts = (steps + p.stretch - 1) / p.stretch;
        }
    }
    return p;
}

size_t matmul_f8_bytes(size_t M, int N, int K) {        // for either type of output
    size_t most = 0;
    for (const bool wide : {false, true}) {
        const PlanF8 p = plan_f8(M, N, K, wide);
        if (p.parts > 1 && p.parts * M * N * sizeof(float) > most) most = p.parts * M * N * sizeof(float);
    }
    return most;
}

// (Parts of bf16 outputs are fp32, and not wide: only the plans that are cut into stretches have that form.  The largest tiles are not wide either: their
// operands would not fit the registers.)
template <typename T, bool WIDE> static hipError_t run_f8(const PlanF8 &plan, ProductF8Args p, size_t M, int N, hipStream_t s, const char **name) {
    const auto count = [](size_t all, unsigned of) { return (unsigned)((all - 1) / of + 1); };
    const auto run = [&](auto kern, const char *name_of) {
        *name = name_of;
        const unsigned bm = plan.bm, bn = plan.bn, most = most_blocks(plan.threads) / plan.parts, nt = count(N, bn) < most ? count(N, bn) : most;
        const size_t m_step = (size_t)(most / nt) * bm, n_step = (size_t)nt * bn;       // of one launch at most
        for (size_t m = 0; m < M; m += m_step)
            for (size_t n = 0; n < (size_t)N; n += n_step) {
                ProductF8Args q = p;
                q.M = M - m < m_step ? M - m : m_step;
                q.N = (int)(N - n < n_step ? N - n : n_step);
                q.a += m * p.pitch, q.a_scale += m * p.s_pitch, q.w += n * p.pitch, q.w_scale += n * p.s_pitch;
                if (p.bias) q.bias += n;
                q.out = static_cast<T *>(p.out) + m * p.ldo + n;
                q.mtiles = count(q.M, bm), q.ntiles = count(q.N, bn), q.tiles = q.mtiles * q.ntiles;
                hipLaunchKernelGGL(kern, dim3(q.tiles * plan.parts), dim3(plan.threads), 0, s, q);
            }
        return hipGetLastError();
    };
    if (plan.kernel == kSmall1) return run(product_f8_small_kernel<T, WIDE, 1, 1, 8, 4>, "product_f8_small<1,1>");
    if (plan.kernel == kTile64) return run(product_f8_tile_kernel<T, WIDE, 2, 4, 1, 1, 3>, "product_f8_tile<64,128>");
    if constexpr (sizeof(T) == 2 || WIDE) {
        if (plan.kernel == kSmall2) return run(product_f8_small_kernel<T, WIDE, 2, 2, 8, 2>, "product_f8_small<2,2>");
        if (plan.kernel == kTile128Deep) return run(product_f8_tile_kernel<T, WIDE, 2, 4, 2, 1, 4>, "product_f8_tile<128,128>");
        if (plan.kernel == kTile128) return run(product_f8_tile_kernel<T, WIDE, 2, 2, 2, 2, 2>, "product_f8_tile<128,128>");
    }
    if constexpr (sizeof(T) == 2)
        if (plan.kernel == kTile256) return run(product_f8_tile_kernel<T, WIDE, 2, 4, 4, 2, 2>, "product_f8_tile<256,256>");
    return hipErrorNotSupported;
}

template <typename T> static hipError_t product(const ProductF8 &in, float *ws, hipStream_t s, const char **name) {
    constexpr bool WIDE = sizeof(T) == 4;
    const PlanF8 plan = plan_f8(in.M, in.N, in.K, WIDE);
    const size_t bytes = in.M * in.N * sizeof(T);
    const int past = bytes >= kPastCaches && (bytes < 2 * kPastCaches || whole_pieces(in.out, in.N * sizeof(T), in.ldo * sizeof(T)));
    ProductF8Args p{in.a, in.a_scale, in.w, in.w_scale, in.bias, in.out, in.M, in.ldo, 0, in.N, f8_pitch(in.K), f8_scale_pitch(in.K), plan.stretch,
                    0, 0, 0, past};
    if (plan.parts == 1) return run_f8<T, WIDE>(plan, p, in.M, in.N, s, name);
    p.bias = nullptr, p.out = ws, p.ldo = in.N, p.part = in.M * in.N, p.past = 0;
    if (const hipError_t e = run_f8<float, WIDE>(plan, p, in.M, in.N, s, name)) return e;
    const unsigned nv = (in.N + 3) / 4, vectors = (unsigned)(in.M * nv);        // (below 256 tiles of at most 2^16 values)
    hipLaunchKernelGGL(product_f8_join_kernel<T>, dim3((vectors + 255) / 256), dim3(256), 0, s, ws, p.part, (unsigned)plan.parts, vectors, in.N, nv,
                       div_magic(nv), in.bias, static_cast<T *>(in.out), in.ldo);
    return hipGetLastError();
}

hipError_t launch_matmul_f8(const ProductF8 &p, void *ws, hipStream_t s, const char **name) {
    return p.out_dtype == GSPC_F32 ? product<float>(p, static_cast<float *>(ws), s, name) : product<uint16_t>(p, static_cast<float *>(ws), s, name);
}

}  // namespace gspc
