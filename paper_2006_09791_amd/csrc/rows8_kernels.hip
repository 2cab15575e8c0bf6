// 8-bit rows: int8 values [rows][pitch] with one fp32 scale per row, written from fp32 or bf16 rows and read back.
#include "tokens.h"
#include "tokens_internal.h"

namespace gspc {

// `width` lanes (a power of two up to a wave) hold one row, lane l the vectors l, l + width, ...  HELD of them per lane stay in
// registers between the maximum and the rounding; HELD = 0: rows of any length, read a second time.  Bound by memory: 2 or 4
// bytes of a value in, one out; 50176 rows of 512 in bf16 14.5 us, 5.3 TB/s.  (Written past the caches, these took 5 us longer to write
// and read back.)
template <typename T, int V, int HELD>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, size_t ldx, unsigned rows, int cols, int width,
                                                            int8_t *__restrict__ q, float *__restrict__ scale) {
    const unsigned row = (blockIdx.x * 256 + threadIdx.x) / width;
    const int lane = threadIdx.x & (width - 1), nv = vectors_of<V>(cols), pitch = rows8_pitch(cols);
    if (row >= rows) return;                       // whole groups of `width` lanes
    x += (size_t)row * ldx;
    q += (size_t)row * pitch;
    unsigned top = 0;
    Raw<T, V> raw[HELD ? HELD : 1];
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + k * width < nv) raw[k] = fetch<V>(x + vector_start<V>(lane + k * width, cols));
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + k * width < nv) {
                float v[V];
                widen(raw[k], v);
#pragma unroll
                for (int e = 0; e < V; ++e) top = max(top, magnitude(v[e]));
            }
    } else {
        for (int i = lane; i < nv; i += width) {
            float v[V];
            widen(fetch<V>(x + vector_start<V>(i, cols)), v);
#pragma unroll
            for (int e = 0; e < V; ++e) top = max(top, magnitude(v[e]));
        }
    }
    const RowCode c = row_code(lanes_umax(top, width));
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k = 0; k < HELD; ++k)
            if (lane + k * width < nv) {
                float v[V];
                widen(raw[k], v);
                store_codes(q + vector_start<V>(lane + k * width, cols), v, c);
            }
    } else {
        for (int i = lane; i < nv; i += width) {
            float v[V];
            widen(fetch<V>(x + vector_start<V>(i, cols)), v);
            store_codes(q + vector_start<V>(i, cols), v, c);
        }
    }
    for (int i = cols + lane; i < pitch; i += width) q[i] = 0;
    if (lane == 0) scale[row] = c.scale;
}

// 50176 rows of 512 to bf16: 13.9 us, 5.5 TB/s.
template <typename T, int V>
__global__ __launch_bounds__(256) void dequantize_rows_kernel(const int8_t *__restrict__ q, const float *__restrict__ scale,
                                                              unsigned rows, int cols, int width, T *__restrict__ x, size_t ldx, int past) {
    const unsigned row = (blockIdx.x * 256 + threadIdx.x) / width;
    const int lane = threadIdx.x & (width - 1), nv = vectors_of<V>(cols);
    if (row >= rows) return;
    q += (size_t)row * rows8_pitch(cols);
    x += (size_t)row * ldx;
    const float s = scale[row];
    for (int i = lane; i < nv; i += width) {
        const int at = vector_start<V>(i, cols);
        float v[V];
        widen(fetch<V>(q + at), v);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] *= s;
        store(x + at, v, past);
    }
}

// Lanes of a row: as many as it has vectors, rounded up to a power of two, at most a wave.
static int lanes_of(int nv) {
    int w = 1;
    while (w < nv && w < kWave) w *= 2;
    return w;
}

// Launches in pieces whose threads are numbered in 31 bits.
template <typename F> static hipError_t in_pieces(size_t rows, int width, const F &launch) {
    const size_t most = 0x40000000u / width;
    for (size_t at = 0; at < rows; at += most) {
        const unsigned n = (unsigned)(rows - at < most ? rows - at : most);
        launch(at, n, dim3((unsigned)(((size_t)n * width + 255) / 256)));
    }
    return hipGetLastError();
}

template <typename T, int V>
static hipError_t quantize(const T *x, size_t ldx, size_t rows, int cols, int8_t *q, float *scale, hipStream_t s) {
    const int nv = vectors_of<V>(cols), width = lanes_of(nv), each = (nv + width - 1) / width;
    const auto kern = each <= 1 ? quantize_rows_kernel<T, V, 1> : each <= 2 ? quantize_rows_kernel<T, V, 2>
                    : each <= 4 ? quantize_rows_kernel<T, V, 4> : each <= 8 ? quantize_rows_kernel<T, V, 8> : quantize_rows_kernel<T, V, 0>;
    const size_t pitch = rows8_pitch(cols);
    return in_pieces(rows, width, [&](size_t at, unsigned n, dim3 grid) {
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, x + at * ldx, ldx, n, cols, width, q + at * pitch, scale + at);
    });
}

template <typename T>
static hipError_t dequantize(const int8_t *q, const float *scale, size_t rows, int cols, T *x, size_t ldx, hipStream_t s) {
    const int nv = cols >= 8 ? vectors_of<8>(cols) : cols, width = lanes_of(nv);
    const auto kern = cols >= 8 ? dequantize_rows_kernel<T, 8> : dequantize_rows_kernel<T, 1>;
    const size_t pitch = rows8_pitch(cols);
    return in_pieces(rows, width, [&](size_t at, unsigned n, dim3 grid) {
        hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, q + at * pitch, scale + at, n, cols, width, x + at * ldx, ldx,
                           sizeof(T) == 2 && cols >= 32 && rows * cols * 2 >= kPastCaches);
    });
}

hipError_t launch_quantize_rows(const void *x, int dtype, size_t ldx, size_t rows, int cols, int8_t *q, float *scale, hipStream_t s) {
    if (dtype == GSPC_F32) {
        const float *p = static_cast<const float *>(x);
        return cols >= 8 ? quantize<float, 8>(p, ldx, rows, cols, q, scale, s) : quantize<float, 1>(p, ldx, rows, cols, q, scale, s);
    }
    const uint16_t *p = static_cast<const uint16_t *>(x);
    return cols >= 8 ? quantize<uint16_t, 8>(p, ldx, rows, cols, q, scale, s) : quantize<uint16_t, 1>(p, ldx, rows, cols, q, scale, s);
}

hipError_t launch_dequantize_rows(const int8_t *q, const float *scale, size_t rows, int cols, void *x, int dtype, size_t ldx,
                                  hipStream_t s) {
    return dtype == GSPC_F32 ? dequantize(q, scale, rows, cols, static_cast<float *>(x), ldx, s)
                             : dequantize(q, scale, rows, cols, static_cast<uint16_t *>(x), ldx, s);
}

}  // namespace gspc
