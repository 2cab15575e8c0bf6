// 8-bit float rows written from dense rows, along the rows, along the columns (the rows of the transpose), or both, and read back.
#include "float8.h"
#include "tokens_internal.h"

namespace gspc {

// Sixteen lanes hold a block of 128 columns, eight each, so that its maximum is four steps over lanes and no LDS.  Bound by memory: 2 or 4 bytes of a
// value in, one out (50176 x 512 in bf16, 77 MB: 13.4 us, 5.8 TB/s; read back 12.7, 6.1 TB/s).
template <typename T, Rows ROWS>
__global__ __launch_bounds__(256) void quantize_f8_kernel(const T *__restrict__ x, size_t ldx, unsigned units, int cols, int blocks,
                                                          unsigned m_blocks, uint8_t *__restrict__ q, uint8_t *__restrict__ scale) {
    const unsigned unit = (blockIdx.x * 256 + threadIdx.x) / 16;
    if (unit >= units) return;                          // all sixteen
    const unsigned row = fast_div_any(unit, blocks, m_blocks);
    const int block = unit - row * blocks, lane = threadIdx.x % 16, at = block * kBlock8 + lane * 8;
    const Place some = place_of(at, cols);
    float v[8];
    widen_some<ROWS>(fetch_some<ROWS, true>(x + row * ldx, some), some, v);
    const unsigned code = block_code(lanes_umax(top_of(v), 16));
    *reinterpret_cast<u32x2 *>(q + (size_t)row * blocks * kBlock8 + at) = f8_codes(v, block_up(code));
    const int pitch = f8_scale_pitch(cols);
    uint8_t *s = scale + (size_t)row * pitch + block;
    if (lane == 0) *s = (uint8_t)code;
    else if (block == blocks - 1 && block + lane < pitch) s[lane] = 0;
}

template <typename T, Rows ROWS>
__global__ __launch_bounds__(256) void dequantize_f8_kernel(const uint8_t *__restrict__ q, const uint8_t *__restrict__ scale, unsigned units, int cols,
                                                            int blocks, unsigned m_blocks, T *__restrict__ x, size_t ldx, int past) {
    const unsigned unit = (blockIdx.x * 256 + threadIdx.x) / 16;
    if (unit >= units) return;
    const unsigned row = fast_div_any(unit, blocks, m_blocks);
    const int block = unit - row * blocks, at = block * kBlock8 + threadIdx.x % 16 * 8;
    if (at >= cols) return;
    const float down = block_down(scale[(size_t)row * f8_scale_pitch(cols) + block]);
    float v[8];
    f8_values(*reinterpret_cast<const u32x2 *>(q + (size_t)row * blocks * kBlock8 + at), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= down;
    store_some<ROWS, true>(x + row * ldx, place_of(at, cols), v, past);
}

// A tile of 128 rows and columns, read once: thread (tx, ty) holds columns 8 tx .. + 7 of rows 4 ty .. + 3.  A row's block is in sixteen
// lanes; a column's is joined through LDS, and so are its codes turned, so that stores are whole lines of either form.  (q or qt may be null.)
// Bound by memory and by its phases, loads, maxima, codes and stores, which overlap only among the four blocks of a compute unit (50176 x 512 in bf16,
// 103 MB: 21.7 us, 4.7 TB/s; 5365 x 333 in fp32: 6.4).  With 256 threads, eight rows each, 13.2 us on the latter in place of 6.4.
template <typename T, Rows ROWS>
__global__ __launch_bounds__(512) void quantize_f8_turned_kernel(const T *__restrict__ x, size_t ldx, unsigned rows, int cols, unsigned first,
                                                                 unsigned m_blocks, uint8_t *__restrict__ q, uint8_t *__restrict__ scale,
                                                                 uint8_t *__restrict__ qt, uint8_t *__restrict__ scale_t) {
    constexpr int TURN = kBlock8 / 4 + 1;               // words of a column in LDS
    __shared__ unsigned s_top[8][kBlock8], s_turn[kBlock8 * TURN];
    const int blocks = f8_pitch(cols) / kBlock8, t = threadIdx.x, tx = t % 16, ty = t / 16;
    const unsigned tile = first + blockIdx.x, row_tile = fast_div_any(tile, blocks, m_blocks);
    const int block = tile - row_tile * blocks, at = block * kBlock8 + tx * 8;
    const Place some = place_of(at, cols);
    const unsigned r0 = row_tile * kBlock8;
    Raw<T, 8> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned row = r0 + ty * 4 + i;
        raw[i] = fetch_some<ROWS, true>(x + (size_t)min(row, rows - 1) * ldx, some);
    }
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) widen_some<ROWS>(raw[i], some, v[i], r0 + ty * 4 + i < rows);
    if (q) {
        const size_t pitch = (size_t)blocks * kBlock8, s_pitch = f8_scale_pitch(cols);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned row = r0 + ty * 4 + i;
            const unsigned code = block_code(lanes_umax(top_of(v[i]), 16));
            if (row < rows) {
                *reinterpret_cast<u32x2 *>(q + row * pitch + at) = f8_codes(v[i], block_up(code));
                uint8_t *s = scale + row * s_pitch + block;
                if (tx == 0) *s = (uint8_t)code;
                else if (block == blocks - 1 && block + tx < (int)s_pitch) s[tx] = 0;
            }
        }
    }
    if (!qt) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {                       // over the four rows of lanes of the wave
        const float column[4] = {v[0][e], v[1][e], v[2][e], v[3][e]};
        const unsigned mine = top_of(column);
        const auto a = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
        const unsigned m = max((unsigned)a[0], (unsigned)a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        if (t % kWave < 16) s_top[t / kWave][tx * 8 + e] = max((unsigned)b[0], (unsigned)b[1]);
    }
    __syncthreads();
    const int r_blocks = (int)((rows + kBlock8 - 1) / kBlock8);
    if (t < kBlock8) {                                  // the columns' powers of two, in the first wave's place
        unsigned top = s_top[0][t];
#pragma unroll
        for (int w = 1; w < 8; ++w) top = max(top, s_top[w][t]);
        const unsigned code = block_code(top);
        s_top[0][t] = code;
        if (block * kBlock8 + t < cols) {
            const int s_pitch = f8_scale_pitch((int)rows);
            uint8_t *s = scale_t + (size_t)(block * kBlock8 + t) * s_pitch + row_tile;
            *s = (uint8_t)code;
            if ((int)row_tile == r_blocks - 1)
                for (int i = 1; (int)row_tile + i < s_pitch; ++i) s[i] = 0;
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = tx * 8 + e;
        const float up = block_up(s_top[0][c]);
        s_turn[c * TURN + ty] = f8_word(v[0][e] * up, v[1][e] * up, v[2][e] * up, v[3][e] * up);
    }
    __syncthreads();
    const size_t pitch_t = (size_t)r_blocks * kBlock8;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = j * 64 + t / 8, piece = t % 8;
        if (block * kBlock8 + c < cols) {
            const unsigned *w = s_turn + c * TURN + piece * 4;
            *reinterpret_cast<u32x4 *>(qt + (size_t)(block * kBlock8 + c) * pitch_t + r0 + piece * 16) = (u32x4){w[0], w[1], w[2], w[3]};
        }
    }
}

// Launches of fewer than 2^32 threads: rows in pieces of at most 2^26 blocks of columns.
template <typename F> static hipError_t by_rows(size_t rows, int blocks, const F &launch) {
    const size_t most = (1u << 26) / blocks;
    for (size_t at = 0; at < rows; at += most) {
        const size_t n = rows - at < most ? rows - at : most;
        launch(at, (unsigned)(n * blocks), dim3((unsigned)((n * blocks + 15) / 16)));
    }
    return hipGetLastError();
}

template <typename T> static hipError_t quantize(const QuantizeF8 &a, hipStream_t s) {
    const T *x = static_cast<const T *>(a.x);
    const int pitch = f8_pitch(a.cols), blocks = pitch / kBlock8, s_pitch = f8_scale_pitch(a.cols);
    const Rows kind = rows_of(a.cols);
    const auto rows_only = kind == kWhole ? quantize_f8_kernel<T, kWhole> : kind == kRagged ? quantize_f8_kernel<T, kRagged> : quantize_f8_kernel<T, kThin>;
    const auto turned = kind == kWhole ? quantize_f8_turned_kernel<T, kWhole>
                      : kind == kRagged ? quantize_f8_turned_kernel<T, kRagged> : quantize_f8_turned_kernel<T, kThin>;
    if (!a.qt)
        return by_rows(a.rows, blocks, [&](size_t at, unsigned units, dim3 grid) {
            hipLaunchKernelGGL(rows_only, grid, dim3(256), 0, s, x + at * a.ldx, a.ldx, units, a.cols, blocks, div_magic(blocks),
                               a.q + at * pitch, a.scale + at * s_pitch);
        });
    const size_t tiles = (a.rows + kBlock8 - 1) / kBlock8 * blocks, most = most_blocks(512);
    for (size_t at = 0; at < tiles; at += most)
        hipLaunchKernelGGL(turned, dim3((unsigned)(tiles - at < most ? tiles - at : most)), dim3(512), 0, s, x, a.ldx,
                           (unsigned)a.rows, a.cols, (unsigned)at, div_magic(blocks), a.q, a.scale, a.qt, a.scale_t);
    return hipGetLastError();
}

template <typename T>
static hipError_t dequantize(const uint8_t *q, const uint8_t *scale, size_t rows, int cols, T *x, size_t ldx, hipStream_t s) {
    const int pitch = f8_pitch(cols), blocks = pitch / kBlock8, s_pitch = f8_scale_pitch(cols);
    const int past = sizeof(T) == 2 && rows * cols * 2 >= kPastCaches && whole_pieces(x, cols * sizeof(T), ldx * sizeof(T));
    const auto kern = cols % 8 == 0 ? dequantize_f8_kernel<T, kWhole> : dequantize_f8_kernel<T, kRagged>;
    return by_rows(rows, blocks, [&](size_t at, unsigned units, dim3 grid) {
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, q + at * pitch, scale + at * s_pitch, units, cols, blocks, div_magic(blocks),
                           x + at * ldx, ldx, past);
    });
}

hipError_t launch_quantize_f8(const QuantizeF8 &a, hipStream_t s) { return a.dtype == GSPC_F32 ? quantize<float>(a, s) : quantize<uint16_t>(a, s); }

hipError_t launch_dequantize_f8(const uint8_t *q, const uint8_t *scale, size_t rows, int cols, void *x, int dtype, size_t ldx, hipStream_t s) {
    return dtype == GSPC_F32 ? dequantize(q, scale, rows, cols, static_cast<float *>(x), ldx, s)
                             : dequantize(q, scale, rows, cols, static_cast<uint16_t *>(x), ldx, s);
}

}  // namespace gspc
