// 8-bit float rows written from dense rows, along the rows, along the columns (the rows of the transpose), or both, and read back.
#include "float8.h"
#include "tokens_internal.h"

namespace gspc {

// Sixteen lanes hold a block of 128 columns, eight each.  Bound by memory: 2 or 4 bytes of a value in, one out.
template <typename T>
__global__ __launch_bounds__(256) void quantize_f8_kernel(const T *__restrict__ x, size_t ldx, unsigned units, int cols, int blocks,
                                                          unsigned m_blocks, uint8_t *__restrict__ q, uint8_t *__restrict__ scale) {
    const unsigned unit = (blockIdx.x * 256 + threadIdx.x) / 16;
    if (unit >= units) return;                          // all sixteen
    const unsigned row = fast_div_any(unit, blocks, m_blocks);
    const int block = unit - row * blocks, lane = threadIdx.x % 16, at = block * kBlock8 + lane * 8;
    float v[8];
    widen(fetch_some(x + row * ldx + at, cols - at), v);
    const unsigned code = block_code(lanes_umax(top_of(v), 16));
    *reinterpret_cast<u32x2 *>(q + (size_t)row * blocks * kBlock8 + at) = f8_codes(v, block_up(code));
    const int pitch = f8_scale_pitch(cols);
    uint8_t *s = scale + (size_t)row * pitch + block;
    if (lane == 0) *s = (uint8_t)code;
    else if (block == blocks - 1 && block + lane < pitch) s[lane] = 0;
}

template <typename T>
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
    store_some(x + row * ldx + at, v, cols - at, past);
}

// A tile of 128 rows and columns, read once: thread (tx, ty) holds columns 8 tx .. + 7 of rows 8 ty .. + 7.  A row's block is in sixteen
// lanes; a column's is joined through LDS, and so are its codes turned, so that stores are whole lines of either form.  (q or qt may be null.)
template <typename T>
__global__ __launch_bounds__(256) void quantize_f8_turned_kernel(const T *__restrict__ x, size_t ldx, unsigned rows, int cols, unsigned first,
                                                                 unsigned m_blocks, uint8_t *__restrict__ q, uint8_t *__restrict__ scale,
                                                                 uint8_t *__restrict__ qt, uint8_t *__restrict__ scale_t) {
    constexpr int TURN = kBlock8 / 4 + 1;               // words of a column in LDS
    __shared__ unsigned s_top[4][kBlock8], s_turn[kBlock8 * TURN];
    const int blocks = f8_pitch(cols) / kBlock8, t = threadIdx.x, tx = t % 16, ty = t / 16;
    const unsigned tile = first + blockIdx.x, row_tile = fast_div_any(tile, blocks, m_blocks);
    const int block = tile - row_tile * blocks, at = block * kBlock8 + tx * 8;
    const unsigned r0 = row_tile * kBlock8;
    Raw<T, 8> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned row = r0 + ty * 8 + i;
        raw[i] = fetch_some(x + (size_t)min(row, rows - 1) * ldx + at, row < rows ? cols - at : 0);
    }
    if (q) {
        const size_t pitch = (size_t)blocks * kBlock8, s_pitch = f8_scale_pitch(cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned row = r0 + ty * 8 + i;
            float v[8];
            widen(raw[i], v);
            const unsigned code = block_code(lanes_umax(top_of(v), 16));
            if (row < rows) {
                *reinterpret_cast<u32x2 *>(q + row * pitch + at) = f8_codes(v, block_up(code));
                uint8_t *s = scale + row * s_pitch + block;
                if (tx == 0) *s = (uint8_t)code;
                else if (block == blocks - 1 && block + tx < (int)s_pitch) s[tx] = 0;
            }
        }
    }
    if (!qt) return;
    unsigned top[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float v[8];
        widen(raw[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top[e] = max(top[e], finite_magnitude(v[e]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {                       // over the four rows of lanes of the wave
        const auto a = __builtin_amdgcn_permlane16_swap(top[e], top[e], false, false);
        const unsigned m = max((unsigned)a[0], (unsigned)a[1]);
        const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        top[e] = max((unsigned)b[0], (unsigned)b[1]);
    }
    if (t % kWave < 16)
#pragma unroll
        for (int e = 0; e < 8; ++e) s_top[t / kWave][tx * 8 + e] = top[e];
    __syncthreads();
    const int r_blocks = (int)((rows + kBlock8 - 1) / kBlock8);
    if (t < kBlock8 && block * kBlock8 + t < cols) {
        const unsigned code = block_code(max(max(s_top[0][t], s_top[1][t]), max(s_top[2][t], s_top[3][t])));
        const int s_pitch = f8_scale_pitch((int)rows);
        uint8_t *s = scale_t + (size_t)(block * kBlock8 + t) * s_pitch + row_tile;
        *s = (uint8_t)code;
        if ((int)row_tile == r_blocks - 1)
            for (int i = 1; (int)row_tile + i < s_pitch; ++i) s[i] = 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = tx * 8 + e;
        const float up = block_up(block_code(max(max(s_top[0][c], s_top[1][c]), max(s_top[2][c], s_top[3][c]))));
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float w[8];
            widen(raw[i], w);
            v[i] = w[e];
        }
        const u32x2 codes = f8_codes(v, up);
        s_turn[c * TURN + ty * 2] = codes[0];
        s_turn[c * TURN + ty * 2 + 1] = codes[1];
    }
    __syncthreads();
    const size_t pitch_t = (size_t)r_blocks * kBlock8;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = j * 32 + t / 8, piece = t % 8;
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
    if (!a.qt)
        return by_rows(a.rows, blocks, [&](size_t at, unsigned units, dim3 grid) {
            hipLaunchKernelGGL(quantize_f8_kernel<T>, grid, dim3(256), 0, s, x + at * a.ldx, a.ldx, units, a.cols, blocks, div_magic(blocks),
                               a.q + at * pitch, a.scale + at * s_pitch);
        });
    const size_t tiles = (a.rows + kBlock8 - 1) / kBlock8 * blocks, most = most_blocks(256);
    for (size_t at = 0; at < tiles; at += most)
        hipLaunchKernelGGL(quantize_f8_turned_kernel<T>, dim3((unsigned)(tiles - at < most ? tiles - at : most)), dim3(256), 0, s, x, a.ldx,
                           (unsigned)a.rows, a.cols, (unsigned)at, div_magic(blocks), a.q, a.scale, a.qt, a.scale_t);
    return hipGetLastError();
}

template <typename T>
static hipError_t dequantize(const uint8_t *q, const uint8_t *scale, size_t rows, int cols, T *x, size_t ldx, hipStream_t s) {
    const int pitch = f8_pitch(cols), blocks = pitch / kBlock8, s_pitch = f8_scale_pitch(cols);
    const int past = sizeof(T) == 2 && rows * cols * 2 >= kPastCaches && whole_pieces(x, cols * sizeof(T), ldx * sizeof(T));
    return by_rows(rows, blocks, [&](size_t at, unsigned units, dim3 grid) {
        hipLaunchKernelGGL(dequantize_f8_kernel<T>, grid, dim3(256), 0, s, q + at * pitch, scale + at * s_pitch, units, cols, blocks, div_magic(blocks),
                           x + at * ldx, ldx, past);
    });
}

hipError_t launch_quantize_f8(const QuantizeF8 &a, hipStream_t s) { return a.dtype == GSPC_F32 ? quantize<float>(a, s) : quantize<uint16_t>(a, s); }

hipError_t launch_dequantize_f8(const uint8_t *q, const uint8_t *scale, size_t rows, int cols, void *x, int dtype, size_t ldx, hipStream_t s) {
    return dtype == GSPC_F32 ? dequantize(q, scale, rows, cols, static_cast<float *>(x), ldx, s)
                             : dequantize(q, scale, rows, cols, static_cast<uint16_t *>(x), ldx, s);
}

}  // namespace gspc
