// Host side shared by the C-ABI sources: the calling thread's stream and error
// message, and the checks of arguments.  Every check runs before any HIP call.
#pragma once

#include "../../include/xdit.h"

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

namespace xdit_api {

inline thread_local hipStream_t g_stream = nullptr;
inline thread_local char g_error[512] = "";

inline int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof(g_error), fmt, ap);
    va_end(ap);
    return code;
}

inline void clear_error() { g_error[0] = '\0'; }

constexpr int64_t kMaxDim = INT32_MAX;

inline int esize_of(int32_t dtype) { return dtype == XDIT_BF16 ? 2 : 4; }

inline int check_dtype_dim(int32_t dtype, int64_t head_dim) {
    if (dtype != XDIT_BF16 && dtype != XDIT_F32)
        return fail(XDIT_ERR_DTYPE, "unknown dtype %d (expected XDIT_BF16=0 or XDIT_F32=1)", dtype);
    if (head_dim != 64 && head_dim != 72 && head_dim != 128)
        return fail(XDIT_ERR_UNSUPPORTED, "head_dim %lld not supported (64, 72 or 128)",
                    (long long)head_dim);
    return XDIT_OK;
}

inline int check_dims(const char* what, int64_t B, int64_t n1, int64_t n2, int64_t H) {
    if (B < 0 || n1 < 0 || n2 < 0 || H < 0)
        return fail(XDIT_ERR_SHAPE, "%s: negative dimension", what);
    if (B > kMaxDim || n1 > kMaxDim || n2 > kMaxDim || H > kMaxDim)
        return fail(XDIT_ERR_SHAPE, "%s: dimension exceeds 2^31-1", what);
    // keep every tensor below 2^40 elements so offsets never overflow
    if ((double)B * (double)(n1 > n2 ? n1 : n2) * (double)H * 128.0 > 1099511627776.0)
        return fail(XDIT_ERR_SHAPE, "%s: tensor too large", what);
    return XDIT_OK;
}

// The kernels address each batch's rows with 32-bit byte offsets, plus up to
// one tile (256 rows) of look-ahead past the end.
inline int check_batch_bytes(const char* what, int64_t rows, int64_t heads, int64_t head_dim, int esize) {
    const int64_t row = heads * head_dim * esize;
    if ((rows + 256) * row >= ((int64_t)1 << 31))
        return fail(XDIT_ERR_SHAPE, "%s: one batch of a tensor exceeds 2 GiB", what);
    return XDIT_OK;
}

struct Span {
    const void* p;
    int64_t bytes;
    const char* name;
};

inline bool overlap(const Span& a, const Span& b) {
    if (a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    return a0 < b0 + (uintptr_t)b.bytes && b0 < a0 + (uintptr_t)a.bytes;
}

inline int check_ptr(const Span& s) {
    if (s.bytes > 0 && s.p == nullptr) return fail(XDIT_ERR_NULL, "%s is NULL", s.name);
    if (s.bytes > 0 && ((uintptr_t)s.p & 15u) != 0)
        return fail(XDIT_ERR_LAYOUT, "%s is not 16-byte aligned", s.name);
    return XDIT_OK;
}

inline int check_no_overlap(const Span& out, const Span& in) {
    if (overlap(out, in)) return fail(XDIT_ERR_ALIAS, "%s overlaps %s", out.name, in.name);
    return XDIT_OK;
}

inline int hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(XDIT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return XDIT_OK;
}

#define XDIT_TRY(expr)            \
    do {                          \
        const int rc_ = (expr);   \
        if (rc_ != XDIT_OK) return rc_; \
    } while (0)

}  // namespace xdit_api
