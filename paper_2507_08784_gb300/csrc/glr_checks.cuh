// What the operators' entry points check their arguments with, and how they refuse and report.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "glr_internal.cuh"

namespace glr {
inline int refuse(const char* fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof(msg), fmt, ap);
    va_end(ap);
    set_global_error(msg);
    return GLR_EINVAL;
}
inline int launched(const char* who, cudaError_t e) {
    if (e == cudaSuccess) return GLR_OK;
    char msg[256];
    snprintf(msg, sizeof(msg), "%s: launch failed: %s", who, cudaGetErrorString(e));
    set_global_error(msg);
    return GLR_ECUDA;
}

inline int64_t bytes_of(int dtype) { return dtype == GLR_BF16 ? 2 : 4; }
inline bool dtype_ok(int dtype) { return dtype == GLR_F32 || dtype == GLR_BF16; }

// A row-major matrix argument: present where it has elements, rows no closer than their length,
// elements on their own size.
inline bool matrix_ok(const void* p, int64_t ld, int64_t rows, int64_t cols, int dtype) {
    if (rows == 0 || cols == 0) return true;
    return p && (rows == 1 || ld >= cols) && reinterpret_cast<uintptr_t>(p) % bytes_of(dtype) == 0;
}
inline bool vector_ok(const void* p, int64_t n, int64_t bytes) {
    return n == 0 || (p && reinterpret_cast<uintptr_t>(p) % bytes == 0);
}
inline bool optional_ok(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

constexpr int64_t kMaxRows = int64_t(1) << 24;

inline bool positive(float x) { return x >= 1.2e-38f && x <= 3.0e38f; }       // its reciprocal too
inline bool finite(float x) { return x >= -3.0e38f && x <= 3.0e38f; }
inline bool flag(int v) { return v == 0 || v == 1; }


}  // namespace glr
