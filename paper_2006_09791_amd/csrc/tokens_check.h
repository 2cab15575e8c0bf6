// Checks of arguments that the entry points of the operators on tokens share.
#pragma once

#include "tokens_internal.h"

namespace gspc {

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxCols = 0x7ffffff0;        // whose pitch is an int

inline int done(hipError_t e, const char *what) {
    return e == hipSuccess ? GSPC_OK : fail(GSPC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool dense(int dtype) { return dtype == GSPC_F32 || dtype == GSPC_BF16; }
inline bool misaligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
inline size_t size_of(int dtype) { return dtype == GSPC_F32 ? 4 : 2; }

// Dense rows of `cols` values: type, stride, alignment.
inline int check_dense(const void *p, int dtype, int64_t ld, int cols, const char *what) {
    if (!dense(dtype)) return fail(GSPC_ERR_DTYPE, "%s: unknown dtype %d", what, dtype);
    if (ld < cols) return fail(GSPC_ERR_DIM, "%s: rows of %d values %lld apart", what, cols, (long long)ld);
    if (misaligned(p, size_of(dtype))) return fail(GSPC_ERR_ARG, "%s must be aligned to its elements", what);
    return GSPC_OK;
}

inline int check_rows8(const void *q, const float *scale, const char *what) {
    if (misaligned(q, 16)) return fail(GSPC_ERR_ARG, "%s: 8-bit rows must be 16-byte aligned", what);
    if (misaligned(scale, 4)) return fail(GSPC_ERR_ARG, "%s: scales must be 4-byte aligned", what);
    return GSPC_OK;
}

inline int check_count(int64_t rows, int cols) {
    if (rows < 0 || rows > kMaxRows) return fail(GSPC_ERR_DIM, "%lld rows", (long long)rows);
    if (cols <= 0 || cols > kMaxCols) return fail(GSPC_ERR_DIM, "%d columns", cols);
    return GSPC_OK;
}

inline int check_workspace(const void *ws, size_t given, size_t needed) {
    if (given < needed) return fail(GSPC_ERR_SPACE, "workspace holds %zu bytes, %zu needed", given, needed);
    if (needed && !ws) return fail(GSPC_ERR_NULL, "null workspace");
    if (misaligned(ws, 16)) return fail(GSPC_ERR_ARG, "workspace must be 16-byte aligned");
    return GSPC_OK;
}

}  // namespace gspc
