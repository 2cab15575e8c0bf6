// Entry points of the channels-last operators: their arguments are checked here, on the host, before anything is launched.
#include <cmath>

#include "divide.h"
#include "tokens_internal.h"

namespace {

using gspc::fail;

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxCols = 0x7ffffff0;        // whose pitch is an int
constexpr int kMaxNormCols = 0x7fffffff - 4096;     // whose slabs of channels end within an int
constexpr int kMaxK = 133144;               // 2^31 / 127^2: sums of products fit 32 bits

int done(hipError_t e, const char *what) {
    return e == hipSuccess ? GSPC_OK : fail(GSPC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool dense(int dtype) { return dtype == GSPC_F32 || dtype == GSPC_BF16; }
bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
size_t size_of(int dtype) { return dtype == GSPC_F32 ? 4 : 2; }

// Dense rows of `cols` values: type, stride, alignment.
int check_dense(const void *p, int dtype, int64_t ld, int cols, const char *what) {
    if (!dense(dtype)) return fail(GSPC_ERR_DTYPE, "%s: unknown dtype %d", what, dtype);
    if (ld < cols) return fail(GSPC_ERR_DIM, "%s: rows of %d values %lld apart", what, cols, (long long)ld);
    if (misaligned(p, size_of(dtype))) return fail(GSPC_ERR_ARG, "%s must be aligned to its elements", what);
    return GSPC_OK;
}

int check_rows8(const void *q, const float *scale, const char *what) {
    if (misaligned(q, 16)) return fail(GSPC_ERR_ARG, "%s: 8-bit rows must be 16-byte aligned", what);
    if (misaligned(scale, 4)) return fail(GSPC_ERR_ARG, "%s: scales must be 4-byte aligned", what);
    return GSPC_OK;
}

int check_count(int64_t rows, int cols) {
    if (rows < 0 || rows > kMaxRows) return fail(GSPC_ERR_DIM, "%lld rows", (long long)rows);
    if (cols <= 0 || cols > kMaxCols) return fail(GSPC_ERR_DIM, "%d columns", cols);
    return GSPC_OK;
}

int check_norm(int N, int P, int C, int groups, int act, gspc::NormShape *h) {
    if (N < 0 || P < 0 || C <= 0 || C > kMaxNormCols) return fail(GSPC_ERR_DIM, "invalid dimension (N=%d P=%d C=%d)", N, P, C);
    if ((int64_t)N * P > kMaxRows) return fail(GSPC_ERR_DIM, "%lld tokens", (long long)N * P);
    if (groups <= 0 || C % groups) return fail(GSPC_ERR_GROUPS, "C=%d must be divisible by groups=%d", C, groups);
    if (act != GSPC_ACT_NONE && act != GSPC_ACT_RELU && act != GSPC_ACT_SILU) return fail(GSPC_ERR_ARG, "unknown activation %d", act);
    if ((int64_t)N * groups > kMaxRows / 64) return fail(GSPC_ERR_DIM, "N * groups = %lld", (long long)N * groups);
    *h = {N, P, C, groups, C / groups, act, gspc::div_magic(C / groups)};
    return GSPC_OK;
}

int check_workspace(const void *ws, size_t given, size_t needed) {
    if (given < needed) return fail(GSPC_ERR_SPACE, "workspace holds %zu bytes, %zu needed", given, needed);
    if (needed && !ws) return fail(GSPC_ERR_NULL, "null workspace");
    if (misaligned(ws, 16)) return fail(GSPC_ERR_ARG, "workspace must be 16-byte aligned");
    return GSPC_OK;
}

int change_layout(const void *in, int in_dtype, int N, int C, int P, void *out, int out_dtype, bool pack) {
    if (N < 0 || P < 0 || C <= 0) return fail(GSPC_ERR_DIM, "invalid dimension (N=%d C=%d P=%d)", N, C, P);
    if (!dense(in_dtype) || !dense(out_dtype)) return fail(GSPC_ERR_DTYPE, "unknown dtype (%d to %d)", in_dtype, out_dtype);
    // (a tile is 64 x 64: with fewer than 2^31 of them the kernel's numbers fit)
    if (((int64_t)C + 63) / 64 * (((int64_t)P + 63) / 64) > kMaxRows) return fail(GSPC_ERR_DIM, "C=%d times P=%d", C, P);
    if (N == 0 || P == 0) return GSPC_OK;
    if (!in || !out) return fail(GSPC_ERR_NULL, "null pointer argument");
    if (misaligned(in, size_of(in_dtype)) || misaligned(out, size_of(out_dtype)))
        return fail(GSPC_ERR_ARG, "tensors must be aligned to their elements");
    gspc::set_last_kernel("transpose");
    return done(gspc::launch_transpose(in, in_dtype, N, pack ? C : P, pack ? P : C, out, out_dtype, gspc::current_stream()),
                "layout launch");
}

}  // namespace

extern "C" {

int gspc_rows8_pitch(int cols) {
    if (cols <= 0 || cols > kMaxCols) {
        fail(GSPC_ERR_DIM, "%d columns", cols);
        return 0;
    }
    return (cols + 15) / 16 * 16;
}

int gspc_pack_channels_last(const void *in, int in_dtype, int N, int C, int P, void *out, int out_dtype) {
    return change_layout(in, in_dtype, N, C, P, out, out_dtype, true);
}

int gspc_unpack_channels_last(const void *in, int in_dtype, int N, int C, int P, void *out, int out_dtype) {
    return change_layout(in, in_dtype, N, C, P, out, out_dtype, false);
}

int gspc_quantize_rows(const void *x, int dtype, int64_t ldx, int64_t rows, int cols, void *q, float *scale) {
    int rc = check_count(rows, cols);
    if (rc || (rc = check_dense(x, dtype, ldx, cols, "x")) || (rc = check_rows8(q, scale, "q"))) return rc;
    if (rows == 0) return GSPC_OK;
    if (!x || !q || !scale) return fail(GSPC_ERR_NULL, "null pointer argument");
    gspc::set_last_kernel("quantize_rows");
    return done(gspc::launch_quantize_rows(x, dtype, ldx, rows, cols, static_cast<int8_t *>(q), scale, gspc::current_stream()),
                "quantize launch");
}

int gspc_dequantize_rows(const void *q, const float *scale, int64_t rows, int cols, void *x, int dtype, int64_t ldx) {
    int rc = check_count(rows, cols);
    if (rc || (rc = check_dense(x, dtype, ldx, cols, "x")) || (rc = check_rows8(q, scale, "q"))) return rc;
    if (rows == 0) return GSPC_OK;
    if (!x || !q || !scale) return fail(GSPC_ERR_NULL, "null pointer argument");
    gspc::set_last_kernel("dequantize_rows");
    return done(gspc::launch_dequantize_rows(static_cast<const int8_t *>(q), scale, rows, cols, x, dtype, ldx, gspc::current_stream()),
                "dequantize launch");
}

size_t gspc_group_norm_workspace_bytes(int N, int P, int C, int groups, int x_dtype, int rows8) {
    gspc::NormShape h;
    if (check_norm(N, P, C, groups, GSPC_ACT_NONE, &h) || (int64_t)N * P == 0) return 0;
    if (!dense(x_dtype)) return fail(GSPC_ERR_DTYPE, "unknown dtype %d", x_dtype), 0;
    return gspc::norm_forward_bytes(h, x_dtype, rows8 != 0, false);
}

size_t gspc_group_norm_backward_workspace_bytes(int N, int P, int C, int groups, int dy_dtype, int x_dtype) {
    gspc::NormShape h;
    if (check_norm(N, P, C, groups, GSPC_ACT_NONE, &h) || (int64_t)N * P == 0) return 0;
    if (!dense(dy_dtype) || (!dense(x_dtype) && x_dtype != GSPC_I8)) return fail(GSPC_ERR_DTYPE, "unknown dtype (%d, %d)", dy_dtype, x_dtype), 0;
    return gspc::norm_backward_bytes(h, dy_dtype);
}

int gspc_group_norm(const void *x, int x_dtype, int64_t ldx, const float *gamma, const float *beta, int N, int P, int C, int groups,
                    float eps, int act, void *y, int y_dtype, int64_t ldy, float *y_scale, float *stats, void *saved,
                    float *saved_scale, void *workspace, size_t workspace_bytes) {
    gspc::NormShape h;
    int rc = check_norm(N, P, C, groups, act, &h);
    if (rc || (rc = check_dense(x, x_dtype, ldx, C, "x"))) return rc;
    if (!(eps > 0.f) || std::isinf(eps)) return fail(GSPC_ERR_ARG, "eps must be positive and finite");
    const bool codes = y_dtype == GSPC_I8;
    if ((rc = codes ? check_rows8(y, y_scale, "y") : check_dense(y, y_dtype, ldy, C, "y"))) return rc;
    if ((rc = check_rows8(saved, saved_scale, "saved"))) return rc;
    if (misaligned(gamma, 4) || misaligned(beta, 4)) return fail(GSPC_ERR_ARG, "gamma and beta must be 4-byte aligned");
    if (misaligned(stats, 8)) return fail(GSPC_ERR_ARG, "stats must be 8-byte aligned");
    if ((int64_t)N * P == 0) return GSPC_OK;
    if (!x || !y || (codes && !y_scale) || (saved && !saved_scale)) return fail(GSPC_ERR_NULL, "null pointer argument");
    if ((rc = check_workspace(workspace, workspace_bytes, gspc::norm_forward_bytes(h, x_dtype, codes || saved, stats != nullptr)))) return rc;
    const gspc::NormForward f = {x, x_dtype, (size_t)ldx, gamma, beta, eps, y, y_dtype, (size_t)ldy, y_scale, stats,
                                 static_cast<int8_t *>(saved), saved_scale, 0};
    const char *name = "";
    const hipError_t e = gspc::launch_norm_forward(h, f, workspace, gspc::current_stream(), &name);
    gspc::set_last_kernel(name);
    return done(e, "group norm launch");
}

int gspc_group_norm_backward(const void *dy, int dy_dtype, int64_t lddy, const void *x, int x_dtype, int64_t ldx, const float *x_scale,
                             const float *stats, const float *gamma, const float *beta, int N, int P, int C, int groups, int act,
                             void *dx, int64_t lddx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes) {
    gspc::NormShape h;
    int rc = check_norm(N, P, C, groups, act, &h);
    if (rc || (rc = check_dense(dy, dy_dtype, lddy, C, "dy")) || (rc = check_dense(dx, dy_dtype, lddx, C, "dx"))) return rc;
    const bool codes = x_dtype == GSPC_I8;
    if ((rc = codes ? check_rows8(x, x_scale, "x") : check_dense(x, x_dtype, ldx, C, "x"))) return rc;
    if (misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(dgamma, 4) || misaligned(dbeta, 4))
        return fail(GSPC_ERR_ARG, "gamma, beta and their gradients must be 4-byte aligned");
    if (misaligned(stats, 8)) return fail(GSPC_ERR_ARG, "stats must be 8-byte aligned");
    if ((int64_t)N * P > 0) {
        if (!dy || !x || !dx || !stats || (codes && !x_scale)) return fail(GSPC_ERR_NULL, "null pointer argument");
        if ((rc = check_workspace(workspace, workspace_bytes, gspc::norm_backward_bytes(h, dy_dtype)))) return rc;
    }
    if (codes) ldx = gspc_rows8_pitch(C);
    const gspc::NormBackward b = {dy, dy_dtype, (size_t)lddy, x, x_dtype, (size_t)ldx, x_scale, stats, gamma, beta,
                                  dx, (size_t)lddx, dgamma, dbeta, 0};
    const char *name = "";
    const hipError_t e = gspc::launch_norm_backward(h, b, workspace, gspc::current_stream(), &name);
    gspc::set_last_kernel(name);
    return done(e, "group norm gradient launch");
}

int gspc_matmul_i8(const void *a, const float *a_scale, const void *w, const float *w_scale, const float *bias, int64_t M, int N, int K,
                   void *out, int out_dtype, int64_t ldo) {
    int rc = check_count(M, N);
    if (rc) return rc;
    if (K <= 0 || K > kMaxK) return fail(GSPC_ERR_DIM, "K=%d (1 .. %d: sums of products fit 32 bits)", K, kMaxK);
    if ((rc = check_dense(out, out_dtype, ldo, N, "out"))) return rc;
    if ((rc = check_rows8(a, a_scale, "a")) || (rc = check_rows8(w, w_scale, "w"))) return rc;
    if (misaligned(bias, 4)) return fail(GSPC_ERR_ARG, "bias must be 4-byte aligned");
    if (M == 0) return GSPC_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return fail(GSPC_ERR_NULL, "null pointer argument");
    if ((double)((M + 15) / 16) * ((N + 15) / 16) > kMaxRows) return fail(GSPC_ERR_DIM, "M=%lld times N=%d", (long long)M, N);
    const gspc::ProductI8 p = {static_cast<const int8_t *>(a), static_cast<const int8_t *>(w), a_scale, w_scale, bias, out,
                               (size_t)M, (size_t)ldo, N, K, out_dtype};
    const char *name = "";
    const hipError_t e = gspc::launch_matmul_i8(p, gspc::current_stream(), &name);
    gspc::set_last_kernel(name);
    return done(e, "8-bit product launch");
}

}  // extern "C"
