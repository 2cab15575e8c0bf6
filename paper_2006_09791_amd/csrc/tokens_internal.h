// Launches of the channels-last operators (tokens_api.cpp calls them with checked arguments).
#pragma once

#include "gspc_internal.h"
#include "philox.h"

namespace gspc {

// The calling thread's stream and error text, which all entry points share (gspc_api.cpp).
hipStream_t current_stream();
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
void set_last_kernel(const char *name);

// Blocks of one launch at most: HIP numbers a dimension's threads, not its blocks, in 32 bits.
constexpr unsigned most_blocks(unsigned threads) { return 0xffffffffu / threads; }

// in [N][R][S] -> out [N][S][R]
hipError_t launch_transpose(const void *in, int in_dtype, int N, int R, int S, void *out, int out_dtype, hipStream_t s);

hipError_t launch_quantize_rows(const void *x, int dtype, size_t ldx, size_t rows, int cols, int8_t *q, float *scale, hipStream_t s);
hipError_t launch_dequantize_rows(const int8_t *q, const float *scale, size_t rows, int cols, void *x, int dtype, size_t ldx,
                                  hipStream_t s);

// Group norm.  Rows of the tensors are tokens, ldX elements apart; image n is the rows n P .. (n + 1) P - 1.
struct NormShape {
    int N, P, C, groups, D, act;    // D = C / groups
    unsigned m_D;                   // div_magic(D)
};
struct NormForward {
    const void *x;
    int x_dtype;
    size_t ldx;
    const float *gamma, *beta;      // nullptr: 1, 0
    float eps;
    void *y;
    int y_dtype;                    // GSPC_F32, GSPC_BF16 or GSPC_I8 (8-bit rows, with y_scale)
    size_t ldy;
    float *y_scale;
    float *stats;                   // [N][groups][2]: mean, 1 / standard deviation
    int8_t *saved;                  // x as 8-bit rows, or nullptr
    float *saved_scale;
    int past;                       // y is stored past the caches (set by the launch)
};
struct NormBackward {
    const void *dy;
    int dy_dtype;                   // of dx too
    size_t lddy;
    const void *x;
    int x_dtype;
    size_t ldx;
    const float *x_scale;
    const float *stats, *gamma, *beta;
    void *dx;
    size_t lddx;
    float *dgamma, *dbeta;          // either may be nullptr
    int past;                       // dx is stored past the caches (set by the launch)
};
// Workspace of a call; rows8: one that writes 8-bit rows; given: one that has the caller's memory for the statistics.
size_t norm_forward_bytes(const NormShape &h, int x_dtype, bool rows8, bool given);
size_t norm_backward_bytes(const NormShape &h, int dy_dtype);
hipError_t launch_norm_forward(const NormShape &h, const NormForward &f, void *ws, hipStream_t s, const char **name);
hipError_t launch_norm_backward(const NormShape &h, const NormBackward &b, void *ws, hipStream_t s, const char **name);

// out[m][n] = a_scale[m] w_scale[n] sum_k a[m][k] w[n][k] + bias[n]
struct ProductI8 {
    const int8_t *a, *w;
    const float *a_scale, *w_scale, *bias;
    void *out;
    size_t M, ldo;
    int N, K, out_dtype;
};
hipError_t launch_matmul_i8(const ProductI8 &p, hipStream_t s, const char **name);

// 8-bit float rows: along the rows (q, scale), along the columns (qt, scale_t), or both
struct QuantizeF8 {
    const void *x;
    int dtype;
    size_t ldx, rows;
    int cols;
    uint8_t *q, *scale, *qt, *scale_t;
};
hipError_t launch_quantize_f8(const QuantizeF8 &a, hipStream_t s);
hipError_t launch_dequantize_f8(const uint8_t *q, const uint8_t *scale, size_t rows, int cols, void *x, int dtype, size_t ldx, hipStream_t s);

// out[m][n] = sum_k a[m][k] w[n][k] + bias[n], both 8-bit float rows
struct ProductF8 {
    const uint8_t *a, *a_scale, *w, *w_scale;
    const float *bias;
    void *out;
    size_t M, ldo;
    int N, K, out_dtype;
};
size_t matmul_f8_bytes(size_t M, int N, int K);
hipError_t launch_matmul_f8(const ProductF8 &p, void *ws, hipStream_t s, const char **name);

hipError_t launch_dropout(const Dropout &d, const void *x, int dtype, size_t ldx, size_t rows, int cols, void *y, size_t ldy, hipStream_t s);

// A block's residual norms: x' = scale x + gate drop(post(h)), z = act(pre(x')).  Rows of the tensors are tokens.
enum { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
struct Residual {
    unsigned rows, gates, gate_rows;        // gate_rows: tokens of each of `gates` gates
    int cols, post, pre, act;
    const float *post_gamma, *post_beta, *pre_gamma, *pre_beta, *gate;      // nullptr: 1, 0, 1, 0, 1
    float scale, eps;
    Dropout drop;
};
struct ResidualForward {
    const void *x;
    int x_dtype;                    // of xo too
    size_t ldx;
    const void *h;                  // or nullptr: x' = scale x
    int h_dtype;
    size_t ldh;
    void *xo;                       // or nullptr
    size_t ldxo;
    void *z;                        // or nullptr
    int z_dtype;                    // GSPC_F32, GSPC_BF16 or GSPC_F8 (8-bit float rows, with z_scale)
    size_t ldz;
    uint8_t *z_scale;
    float *stats;                   // [rows][4]: mean and 1 / deviation of h, then of x'; or nullptr
    int past;                       // xo and z are stored past the caches (set by the launch)
};
struct ResidualBackward {
    const void *dz;                 // or nullptr
    int dz_dtype;
    size_t lddz;
    const void *dxo;                // type of x; or nullptr
    size_t lddxo;
    const void *xo;
    int x_dtype;
    size_t ldxo;
    const void *h;
    int h_dtype;                    // of dh too
    size_t ldh;
    const float *stats;
    void *dx;
    size_t lddx;
    void *dh;
    size_t lddh;
    float *dgate, *dpost_gamma, *dpost_beta, *dpre_gamma, *dpre_beta;       // any may be nullptr
    int past, has_dz, has_dxo, has_h;   // (set by the launch)
};
size_t residual_grad_bytes(const Residual &a);
hipError_t launch_residual_norm(const Residual &a, ResidualForward f, hipStream_t s);
hipError_t launch_residual_grad(const Residual &a, ResidualBackward f, void *ws, hipStream_t s);

}  // namespace gspc
