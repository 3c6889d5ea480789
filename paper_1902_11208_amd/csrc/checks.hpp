// Argument checks that the host files of the sequence operators share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "host.hpp"
#include "mdlstm.h"

namespace {

[[maybe_unused]] mdlstm_status fail(mdlstm_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return mdl::set_error(st, buf);
}

#define HIP_OR_FAIL(expr)                                                                                   \
    do {                                                                                                    \
        hipError_t _e = (expr);                                                                             \
        if (_e != hipSuccess) return fail(MDLSTM_ERR_DEVICE, "%s: %s", #expr, hipGetErrorString(_e));       \
    } while (0)

#define OK_OR_RETURN(expr)                        \
    do {                                          \
        const mdlstm_status _st = (expr);         \
        if (_st != MDLSTM_OK) return _st;         \
    } while (0)

constexpr int64_t kMaxTokens = (int64_t)1 << 35;  // products with a dimension or a head count stay within int64
constexpr int64_t kMaxStride = (int64_t)1 << 62;

[[maybe_unused]] size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
[[maybe_unused]] bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
[[maybe_unused]] size_t element(int32_t dtype) { return dtype == MDLSTM_BF16 ? 2 : 4; }

[[maybe_unused]] mdlstm_status check_dtype(int32_t dtype) {
    if (dtype != MDLSTM_F32 && dtype != MDLSTM_BF16)
        return fail(MDLSTM_ERR_INVALID_ARG, "dtype %d is not MDLSTM_F32 or MDLSTM_BF16", dtype);
    return MDLSTM_OK;
}

[[maybe_unused]] mdlstm_status check_sequences(int32_t n, int64_t tokens, int64_t longest) {
    if (n < 0 || n > MDLSTM_MAX_RECTS) return fail(MDLSTM_ERR_INVALID_ARG, "%d examples: 0 to %d", n, MDLSTM_MAX_RECTS);
    if (tokens < 0 || tokens > kMaxTokens || longest < 0 || longest > tokens)
        return fail(MDLSTM_ERR_INVALID_ARG, "%lld tokens, the longest example %lld", (long long)tokens, (long long)longest);
    if (n == 0 && tokens > 0) return fail(MDLSTM_ERR_INVALID_ARG, "%lld tokens of no example", (long long)tokens);
    return MDLSTM_OK;
}

[[maybe_unused]] mdlstm_status check_out(const void* p, const char* name, bool needed, size_t to) {
    if (needed && !p) return fail(MDLSTM_ERR_INVALID_ARG, "%s is NULL", name);
    if (misaligned(p, to)) return fail(MDLSTM_ERR_INVALID_ARG, "%s must be %zu-byte aligned", name, to);
    return MDLSTM_OK;
}

// The bytes of an argument, and whether the call writes them.
struct Span {
    const char* name;
    uintptr_t from, size;
    bool written;
};
[[maybe_unused]] Span span(const char* name, const void* p, int64_t bytes, bool written) {
    return Span{name, reinterpret_cast<uintptr_t>(p), p ? (uintptr_t)bytes : 0, written};
}
// Nothing that the call writes may overlap anything else: workgroups read and write in no order.
template <size_t N>
[[maybe_unused]] mdlstm_status check_apart(const Span (&s)[N]) {
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < N && s[i].written; ++j)
            if (j != i && s[i].size && s[j].size && s[i].from < s[j].from + s[j].size && s[j].from < s[i].from + s[i].size)
                return fail(MDLSTM_ERR_INVALID_ARG, "%s overlaps %s", s[i].name, s[j].name);
    return MDLSTM_OK;
}

[[maybe_unused]] mdlstm_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws || have < need) return fail(MDLSTM_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws ? have : 0, need);
    if (misaligned(ws, 16)) return fail(MDLSTM_ERR_INVALID_ARG, "the workspace must be 16-byte aligned");
    return MDLSTM_OK;
}

[[maybe_unused]] mdlstm_status check_rows(const void* p, const char* name, int64_t rows, int64_t cols, int64_t stride, int32_t dtype) {
    if (rows > 0 && cols > 0 && !p) return fail(MDLSTM_ERR_INVALID_ARG, "%s is NULL", name);
    if (misaligned(p, element(dtype))) return fail(MDLSTM_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    int64_t a;
    if (stride < cols || __builtin_mul_overflow(stride, rows, &a) || a > kMaxStride / 4)
        return fail(MDLSTM_ERR_INVALID_ARG, "rows of %s are %lld elements apart, %lld long", name, (long long)stride,
                    (long long)cols);
    return MDLSTM_OK;
}

}  // namespace
