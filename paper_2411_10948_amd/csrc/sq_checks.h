// Argument checks that the C entry points of the layers share: synchronous,
// before any launch.  Not part of the public ABI; see include/shiftquant.h.
#pragma once

#include <cstdint>
#include <string>

#include "sq_mx.h"

#define SQ_TRY(expr)                      \
    do {                                  \
        const sq_status st__ = (expr);    \
        if (st__ != SQ_OK) return st__;   \
    } while (0)

namespace sq {

constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxCols = (int64_t)1 << 20;
constexpr int64_t kMaxInner = (int64_t)1 << 23;     // a product's inner axis: a tile's 16 groups, 8 bytes an element, in 31 bits
constexpr int64_t kMaxExperts = (int64_t)1 << 16;
constexpr double kMaxBlocks = 2147483647.0;         // of one launch

// No exception leaves a C entry point (a message that cannot be allocated).
template <class F>
inline sq_status guarded(F f) noexcept {
    try {
        return f();
    } catch (...) {
        return SQ_ERR_HIP;
    }
}

inline sq_status invalid(const std::string& msg) { return fail(SQ_ERR_INVALID_ARGUMENT, msg); }

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline sq_status check_type(int32_t type) {
    if (type != SQ_TYPE_F32 && type != SQ_TYPE_BF16) return invalid("type must be SQ_TYPE_F32 or SQ_TYPE_BF16");
    return SQ_OK;
}

inline sq_status check_dim(int64_t n, int64_t limit, const char* name) {
    if (n < 0 || n >= limit) return invalid(std::string(name) + " is out of range");
    return SQ_OK;
}

// a matrix of fp32 or bf16 values that is read or written (its sizes are not 0)
inline sq_status check_values(const void* p, int32_t type, int64_t ld, int64_t cols, const char* name) {
    if (!p) return invalid(std::string(name) + " is NULL");
    if (!aligned(p, type == SQ_TYPE_F32 ? 4 : 2)) return invalid(std::string(name) + " is not aligned to its type");
    if (ld < cols) return invalid(std::string("the row stride of ") + name + " is smaller than its row");
    return SQ_OK;
}

// an array of 32-bit values
inline sq_status check_words(const void* p, const char* name) {
    if (!p || !aligned(p, 4)) return invalid(std::string(name) + " is NULL or misaligned");
    return SQ_OK;
}

inline sq_status check_mx(const void* codes, const void* scales, const char* name) {
    if (!codes || !scales) return invalid(std::string(name) + ": codes or scales are NULL");
    if (!aligned(codes, 16) || !aligned(scales, 4))
        return invalid(std::string(name) + ": codes must be 16-byte and scales 4-byte aligned");
    return SQ_OK;
}

inline sq_status check_inner(int64_t k) {
    if (k >= kMaxInner) return fail(SQ_ERR_UNSUPPORTED, "the inner axis has 2^23 elements or more");
    return SQ_OK;
}

// blocks of the smallest tile that the call's launch may take
inline sq_status check_blocks(int64_t M, int64_t m, int64_t N, int64_t n, int64_t more, int64_t times) {
    if (((double)(M / m) + 1.0 + (double)more) * ((double)(N / n) + 1.0) * (double)times >= kMaxBlocks)
        return fail(SQ_ERR_UNSUPPORTED, "too many tiles for one launch");
    return SQ_OK;
}

inline sq_status check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return SQ_OK;
    if (!ws || !aligned(ws, 16)) return invalid("workspace is NULL or misaligned");
    if (have < need) return fail(SQ_ERR_WORKSPACE_TOO_SMALL, "workspace too small");
    return SQ_OK;
}

}  // namespace sq
