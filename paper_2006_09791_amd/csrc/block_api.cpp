// Entry points of a residual block's operators on tokens - 8-bit float rows and their products, norms with gate and residual, dropout: their
// arguments are checked here, on the host, before anything is launched.
#include <cmath>

#include "tokens_check.h"

namespace {

using namespace gspc;

constexpr int kMaxF8 = 0x7ffffc00;          // columns (or rows, of the turned form) whose pitches are ints
constexpr int kMaxF8K = 1 << 22;            // rows of a product: 256 of them are within 2^30 bytes
constexpr int kMaxResidual = 8192;          // channels: a token is held by 1024 lanes

int check_f8(const void *q, const void *scale, const char *what) {
    if (misaligned(q, 16)) return fail(GSPC_ERR_ARG, "%s: 8-bit float rows must be 16-byte aligned", what);
    if (misaligned(scale, 4)) return fail(GSPC_ERR_ARG, "%s: scales must be 4-byte aligned", what);
    return GSPC_OK;
}

int check_f8_count(int64_t rows, int cols) {
    if (rows < 0 || rows > kMaxRows) return fail(GSPC_ERR_DIM, "%lld rows", (long long)rows);
    if (cols <= 0 || cols > kMaxF8) return fail(GSPC_ERR_DIM, "%d columns", cols);
    return GSPC_OK;
}

int check_dropout(double drop, const uint64_t *step, uint64_t seed, uint64_t offset, Dropout *d) {
    if (!(drop >= 0 && drop <= 1)) return fail(GSPC_ERR_ARG, "a probability of %g", drop);
    if (misaligned(step, 8)) return fail(GSPC_ERR_ARG, "step must be 8-byte aligned");
    const uint32_t limit = (uint32_t)std::nearbyint(drop * 65536);
    *d = {seed, offset, step, limit, limit < 65536 ? 65536.f / (float)(65536 - limit) : 0.f};
    return GSPC_OK;
}

bool norm_kind(int kind) { return kind == GSPC_NORM_NONE || kind == GSPC_NORM_RMS || kind == GSPC_NORM_LAYER; }

// What is common to the forward call and the gradient.
int check_residual(const gspc_residual_t *r, bool h, bool forward, Residual *a) {
    if (!r) return fail(GSPC_ERR_NULL, "null description");
    if (r->rows < 0 || r->rows > kMaxRows) return fail(GSPC_ERR_DIM, "%lld tokens", (long long)r->rows);
    if (r->cols <= 0 || r->cols > kMaxResidual) return fail(GSPC_ERR_DIM, "%d channels (1 .. %d)", r->cols, kMaxResidual);
    if (!norm_kind(r->post) || !norm_kind(r->pre)) return fail(GSPC_ERR_ARG, "unknown norm (%d, %d)", r->post, r->pre);
    if (r->act != GSPC_ACT_NONE && r->act != GSPC_ACT_RELU && r->act != GSPC_ACT_SILU) return fail(GSPC_ERR_ARG, "unknown activation %d", r->act);
    if (r->post == GSPC_NORM_NONE && (r->post_gamma || r->post_beta)) return fail(GSPC_ERR_ARG, "parameters of no norm of h");
    if (r->pre == GSPC_NORM_NONE && (r->pre_gamma || r->pre_beta || r->act != GSPC_ACT_NONE))
        return fail(GSPC_ERR_ARG, "parameters or an activation of no norm of the sum");
    if (forward && (r->post != GSPC_NORM_NONE || r->pre != GSPC_NORM_NONE) && (!(r->eps > 0.f) || std::isinf(r->eps)))
        return fail(GSPC_ERR_ARG, "eps must be positive and finite");
    if (misaligned(r->post_gamma, 4) || misaligned(r->post_beta, 4) || misaligned(r->pre_gamma, 4) || misaligned(r->pre_beta, 4) || misaligned(r->gate, 4))
        return fail(GSPC_ERR_ARG, "parameters and gates must be 4-byte aligned");
    Dropout drop;
    if (const int rc = check_dropout(r->drop, r->step, r->seed, r->offset, &drop)) return rc;
    if (!h && (r->post != GSPC_NORM_NONE || r->gate || drop.limit)) return fail(GSPC_ERR_ARG, "a norm, gate or dropout of no h");
    const int64_t gates = r->gate ? r->gates : 1;
    if (gates <= 0 || r->rows % gates) return fail(GSPC_ERR_GROUPS, "%lld tokens must be divisible by %lld gates", (long long)r->rows, (long long)gates);
    if (gates > kMaxRows) return fail(GSPC_ERR_DIM, "%lld gates", (long long)gates);
    *a = {(unsigned)r->rows, (unsigned)gates, (unsigned)(r->rows / gates), r->cols, r->post, r->pre, r->act, r->post_gamma, r->post_beta, r->pre_gamma,
          r->pre_beta, r->gate, r->scale, r->eps, drop};
    return GSPC_OK;
}

}  // namespace

extern "C" {

int gspc_f8_pitch(int cols) {
    if (cols <= 0 || cols > kMaxF8) {
        fail(GSPC_ERR_DIM, "%d columns", cols);
        return 0;
    }
    return (cols + 127) / 128 * 128;
}

int gspc_f8_scale_pitch(int cols) {
    if (cols <= 0 || cols > kMaxF8) {
        fail(GSPC_ERR_DIM, "%d columns", cols);
        return 0;
    }
    return (cols + 511) / 512 * 4;
}

int gspc_quantize_rows_f8(const void *x, int dtype, int64_t ldx, int64_t rows, int cols, void *q, uint8_t *scale, void *qt, uint8_t *scale_t) {
    int rc = check_f8_count(rows, cols);
    if (rc || (rc = check_dense(x, dtype, ldx, cols, "x")) || (rc = check_f8(q, scale, "q")) || (rc = check_f8(qt, scale_t, "qt"))) return rc;
    if (qt && rows > kMaxF8) return fail(GSPC_ERR_DIM, "%lld rows", (long long)rows);
    if (qt && (rows + 127) / 128 * ((cols + (int64_t)127) / 128) > kMaxRows) return fail(GSPC_ERR_DIM, "%lld rows of %d columns", (long long)rows, cols);
    if (rows == 0) return GSPC_OK;
    if (!x || (!q && !qt) || (q && !scale) || (qt && !scale_t)) return fail(GSPC_ERR_NULL, "null pointer argument");
    set_last_kernel(qt ? "quantize_f8_turned" : "quantize_f8");
    const QuantizeF8 a = {x, dtype, (size_t)ldx, (size_t)rows, cols, static_cast<uint8_t *>(q), scale, static_cast<uint8_t *>(qt), scale_t};
    return done(launch_quantize_f8(a, current_stream()), "quantize launch");
}

int gspc_dequantize_rows_f8(const void *q, const uint8_t *scale, int64_t rows, int cols, void *x, int dtype, int64_t ldx) {
    int rc = check_f8_count(rows, cols);
    if (rc || (rc = check_dense(x, dtype, ldx, cols, "x")) || (rc = check_f8(q, scale, "q"))) return rc;
    if (rows == 0) return GSPC_OK;
    if (!x || !q || !scale) return fail(GSPC_ERR_NULL, "null pointer argument");
    set_last_kernel("dequantize_f8");
    return done(launch_dequantize_f8(static_cast<const uint8_t *>(q), scale, rows, cols, x, dtype, ldx, current_stream()), "dequantize launch");
}

size_t gspc_matmul_f8_workspace_bytes(int64_t M, int N, int K) {
    if (M < 0 || M > kMaxRows || N <= 0 || K <= 0 || K > kMaxF8K) return fail(GSPC_ERR_DIM, "M=%lld N=%d K=%d", (long long)M, N, K), 0;
    return M ? matmul_f8_bytes(M, N, K) : 0;
}

int gspc_matmul_f8(const void *a, const uint8_t *a_scale, const void *w, const uint8_t *w_scale, const float *bias, int64_t M, int N, int K,
                   void *out, int out_dtype, int64_t ldo, void *workspace, size_t workspace_bytes) {
    int rc = check_count(M, N);
    if (rc) return rc;
    if (K <= 0 || K > kMaxF8K) return fail(GSPC_ERR_DIM, "K=%d (1 .. %d)", K, kMaxF8K);
    if ((rc = check_dense(out, out_dtype, ldo, N, "out"))) return rc;
    if ((rc = check_f8(a, a_scale, "a")) || (rc = check_f8(w, w_scale, "w"))) return rc;
    if (misaligned(bias, 4)) return fail(GSPC_ERR_ARG, "bias must be 4-byte aligned");
    if (M == 0) return GSPC_OK;
    if (!a || !a_scale || !w || !w_scale || !out) return fail(GSPC_ERR_NULL, "null pointer argument");
    if ((double)((M + 15) / 16) * ((N + (int64_t)15) / 16) > kMaxRows) return fail(GSPC_ERR_DIM, "M=%lld times N=%d", (long long)M, N);
    if ((rc = check_workspace(workspace, workspace_bytes, matmul_f8_bytes(M, N, K)))) return rc;
    const ProductF8 p = {static_cast<const uint8_t *>(a), a_scale, static_cast<const uint8_t *>(w), w_scale, bias, out, (size_t)M, (size_t)ldo, N, K,
                         out_dtype};
    const char *name = "";
    const hipError_t e = launch_matmul_f8(p, workspace, current_stream(), &name);
    set_last_kernel(name);
    return done(e, "8-bit float product launch");
}

int gspc_dropout(const void *x, int dtype, int64_t ldx, int64_t rows, int cols, double drop, uint64_t seed, uint64_t offset, const uint64_t *step,
                 void *y, int64_t ldy) {
    Dropout d;
    int rc = check_count(rows, cols);
    if (rc || (rc = check_dense(x, dtype, ldx, cols, "x")) || (rc = check_dense(y, dtype, ldy, cols, "y"))) return rc;
    if ((rc = check_dropout(drop, step, seed, offset, &d))) return rc;
    if (rows == 0) return GSPC_OK;
    if (!x || !y) return fail(GSPC_ERR_NULL, "null pointer argument");
    if (x == y && ldx != ldy) return fail(GSPC_ERR_ARG, "rows in place must keep their distance");
    set_last_kernel("dropout");
    return done(launch_dropout(d, x, dtype, ldx, rows, cols, y, ldy, current_stream()), "dropout launch");
}

int gspc_residual_norm(const gspc_residual_t *r, const void *x, int x_dtype, int64_t ldx, const void *h, int h_dtype, int64_t ldh, void *xo,
                       int64_t ldxo, void *z, int z_dtype, int64_t ldz, uint8_t *z_scale, float *stats) {
    Residual a;
    int rc = check_residual(r, h || (r && r->rows == 0), true, &a);
    if (rc || (rc = check_dense(x, x_dtype, ldx, a.cols, "x"))) return rc;
    if (h && (rc = check_dense(h, h_dtype, ldh, a.cols, "h"))) return rc;
    if (xo && (rc = check_dense(xo, x_dtype, ldxo, a.cols, "xo"))) return rc;
    const bool codes = z_dtype == GSPC_F8;
    if (z && (rc = codes ? check_f8(z, z_scale, "z") : check_dense(z, z_dtype, ldz, a.cols, "z"))) return rc;
    if (z && a.pre == GSPC_NORM_NONE) return fail(GSPC_ERR_ARG, "z of no norm");
    if (misaligned(stats, 16)) return fail(GSPC_ERR_ARG, "stats must be 16-byte aligned");
    if (a.rows == 0) return GSPC_OK;
    if (!x || (!xo && !z) || (z && codes && !z_scale)) return fail(GSPC_ERR_NULL, "null pointer argument");
    if (xo == x && ldxo != ldx) return fail(GSPC_ERR_ARG, "rows in place must keep their distance");
    const ResidualForward f = {x, x_dtype, (size_t)ldx, h, h ? h_dtype : x_dtype, (size_t)ldh, xo, (size_t)ldxo, z, z ? z_dtype : GSPC_F32, (size_t)ldz,
                               z_scale, stats, 0};
    if (!z && !stats) a.pre = kNormNone;            // nobody reads it
    set_last_kernel("residual_norm");
    return done(launch_residual_norm(a, f, current_stream()), "residual norm launch");
}

size_t gspc_residual_norm_backward_workspace_bytes(int64_t rows, int cols, int64_t gates) {
    if (rows < 0 || rows > kMaxRows || cols <= 0 || cols > kMaxResidual || gates <= 0 || rows % gates || gates > kMaxRows)
        return fail(GSPC_ERR_DIM, "%lld tokens of %d channels, %lld gates", (long long)rows, cols, (long long)gates), 0;
    Residual a{};
    a.rows = (unsigned)rows, a.cols = cols, a.gates = (unsigned)gates, a.gate_rows = (unsigned)(rows / gates);
    return residual_grad_bytes(a);
}

int gspc_residual_norm_backward(const gspc_residual_t *r, const void *dz, int dz_dtype, int64_t lddz, const void *dxo, int64_t lddxo,
                                const void *xo, int x_dtype, int64_t ldxo, const void *h, int h_dtype, int64_t ldh, const float *stats, void *dx,
                                int64_t lddx, void *dh, int64_t lddh, float *dgate, float *dpost_gamma, float *dpost_beta, float *dpre_gamma,
                                float *dpre_beta, void *workspace, size_t workspace_bytes) {
    Residual a;
    int rc = check_residual(r, h || (r && r->rows == 0), false, &a);
    if (rc || (rc = check_dense(dx, x_dtype, lddx, a.cols, "dx"))) return rc;
    if (dz && ((rc = check_dense(dz, dz_dtype, lddz, a.cols, "dz")) || (rc = check_dense(xo, x_dtype, ldxo, a.cols, "xo")))) return rc;
    if (dxo && (rc = check_dense(dxo, x_dtype, lddxo, a.cols, "dxo"))) return rc;
    if (h && ((rc = check_dense(h, h_dtype, ldh, a.cols, "h")) || (rc = check_dense(dh, h_dtype, lddh, a.cols, "dh")))) return rc;
    if (dz && a.pre == GSPC_NORM_NONE) return fail(GSPC_ERR_ARG, "dz of no norm");
    if ((dpre_gamma || dpre_beta) && a.pre == GSPC_NORM_NONE) return fail(GSPC_ERR_ARG, "gradients of parameters of no norm of the sum");
    if ((dpost_gamma || dpost_beta) && a.post == GSPC_NORM_NONE) return fail(GSPC_ERR_ARG, "gradients of parameters of no norm of h");
    if (dgate && !a.gate) return fail(GSPC_ERR_ARG, "gradient of no gate");
    if (misaligned(stats, 16)) return fail(GSPC_ERR_ARG, "stats must be 16-byte aligned");
    for (const float *p : {dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta})
        if (misaligned(p, 4)) return fail(GSPC_ERR_ARG, "gradients of parameters must be 4-byte aligned");
    if (a.rows) {
        if (!dx || (!dz && !dxo) || (dz && !xo) || (h && !dh) || !stats) return fail(GSPC_ERR_NULL, "null pointer argument");
        if ((dx == dxo && lddx != lddxo) || (h && dh == h && lddh != ldh))
            return fail(GSPC_ERR_ARG, "rows in place must keep their distance");
        if ((rc = check_workspace(workspace, workspace_bytes, residual_grad_bytes(a)))) return rc;
    }
    const ResidualBackward f = {dz, dz_dtype, (size_t)lddz, dxo, (size_t)lddxo, xo, x_dtype, (size_t)ldxo, h, h ? h_dtype : x_dtype, (size_t)ldh, stats,
                                dx, (size_t)lddx, dh, (size_t)lddh, dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta, 0};
    set_last_kernel("residual_grad");
    return done(launch_residual_grad(a, f, workspace, current_stream()), "residual norm gradient launch");
}

}  // extern "C"
