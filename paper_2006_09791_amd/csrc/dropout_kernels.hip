// Dropout of dense rows, forward and gradient: y = x up where the value's sixteen bits are no less than the limit, else 0.
#include "float8.h"
#include "dropout.h"
#include "tokens_internal.h"

namespace gspc {

// A lane has eight columns of a row at a time: one counter of the generator, one vector of memory.  Bound by memory and by its ten rounds at once: twenty
// products of 32 by 32 bits, which take four times as long as other instructions, are half of some 120 instructions' time (200704 x 256 in bf16,
// 206 MB: 36.0 us, 5.7 TB/s).
template <typename T, Rows ROWS>
__global__ __launch_bounds__(256) void dropout_kernel(Dropout d, const T *x, size_t ldx, unsigned first, unsigned vectors, int cols, unsigned nv,
                                                      unsigned m_nv, T *y, size_t ldy, int past) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i >= vectors) return;
    const unsigned row = fast_div_any(i, nv, m_nv), vec = i - row * nv;
    const Place at = place_of(vec * 8, cols);
    const Raw<T, 8> raw = fetch_some<ROWS, true>(x + row * ldx, at);
    const uint64_t call = d.offset + (d.step ? *d.step : 0);
    float v[8];
    widen_some<ROWS>(raw, at, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= d.up;
    drop_some(d, call, first + row, vec, v);
    store_some<ROWS, true>(y + row * ldy, at, v, past);
}

template <typename T> static hipError_t dropout(const Dropout &d, const T *x, size_t ldx, size_t rows, int cols, T *y, size_t ldy, hipStream_t s) {
    const unsigned nv = (cols + 7) / 8;
    const size_t most = (1u << 30) / nv;                // vectors of a launch
    const Rows kind = rows_of(cols);
    const auto kern = kind == kWhole ? dropout_kernel<T, kWhole> : kind == kRagged ? dropout_kernel<T, kRagged> : dropout_kernel<T, kThin>;
    const int past = sizeof(T) == 2 && rows * cols * 2 >= kPastCaches && whole_pieces(y, cols * sizeof(T), ldy * sizeof(T));
    for (size_t at = 0; at < rows; at += most) {
        const size_t n = (rows - at < most ? rows - at : most) * nv;
        hipLaunchKernelGGL(kern, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, d, x + at * ldx, ldx, (unsigned)at, (unsigned)n, cols, nv,
                           div_magic(nv), y + at * ldy, ldy, past);
    }
    return hipGetLastError();
}

hipError_t launch_dropout(const Dropout &d, const void *x, int dtype, size_t ldx, size_t rows, int cols, void *y, size_t ldy, hipStream_t s) {
    return dtype == GSPC_F32 ? dropout(d, static_cast<const float *>(x), ldx, rows, cols, static_cast<float *>(y), ldy, s)
                             : dropout(d, static_cast<const uint16_t *>(x), ldx, rows, cols, static_cast<uint16_t *>(y), ldy, s);
}

}  // namespace gspc
