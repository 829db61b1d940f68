// What the C entry points of the operators share: errors with their message, and checks.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "gefen.h"
#include "ffn_plan.h"
#include "gefen_internal.h"

namespace gefen {

__attribute__((format(printf, 2, 3))) inline int fail(int code, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_last_error(buf);
    return code;
}

#define GEFEN_HIP(call)                                                                  \
    do {                                                                                 \
        hipError_t e_ = (call);                                                          \
        if (e_ != hipSuccess)                                                            \
            return fail(GEFEN_EHIP, "%s failed: %s", #call, hipGetErrorString(e_));      \
    } while (0)

inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

constexpr int64_t kMaxElems = int64_t(1) << 40;

inline int check_rows(int64_t rows, int64_t cols, int64_t max_cols)
{
    if (rows < 0) return fail(GEFEN_EINVAL, "rows must not be negative");
    if (cols < 1 || cols > max_cols)
        return fail(GEFEN_EINVAL, "cols must be in [1, %lld]", (long long)max_cols);
    if (rows > kMaxElems / cols) return fail(GEFEN_EINVAL, "more than 2^40 elements");
    return GEFEN_OK;
}

inline int check_dtype(int32_t dtype)
{
    if (dtype != GEFEN_F32 && dtype != GEFEN_BF16)
        return fail(GEFEN_EDTYPE, "dtype must be GEFEN_F32 or GEFEN_BF16");
    return GEFEN_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename P>
P* at(void* ws, int64_t off)
{
    return reinterpret_cast<P*>(static_cast<char*>(ws) + off);
}

inline int check_space(const void* ws, int64_t have, int64_t need)
{
    if (need > 0 && (!ws || have < need))
        return fail(GEFEN_EINVAL, "workspace of %lld bytes, %lld needed", (long long)have,
                    (long long)need);
    if (!aligned16(ws)) return fail(GEFEN_EINVAL, "workspace must be 16-byte aligned");
    return GEFEN_OK;
}

}  // namespace gefen
