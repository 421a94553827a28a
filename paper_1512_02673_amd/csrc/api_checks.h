// What the C entry points for matrices in few bits, dropout and embeddings ask of their arguments.
#pragma once

#include <algorithm>
#include <exception>
#include <new>

#include "internal.h"

namespace coded {
namespace {

template <class F>
coded_status guarded(F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return fail(CODED_ERR_ARG, "host allocation failed");
    } catch (...) {
        return fail(CODED_ERR_ARG, "unexpected host exception");
    }
}

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int64_t kMostSize = int64_t(1) << 40;

coded_status check_dense(const char* name, coded_dtype dt, const void* p, int64_t rows, int64_t cols, int64_t ld) {
    const std::string what(name);
    if (dt != CODED_F32 && dt != CODED_BF16) return fail(CODED_ERR_ARG, what + " must be CODED_F32 or CODED_BF16");
    if (ld < std::max<int64_t>(cols, 1)) return fail(CODED_ERR_SHAPE, what + ": the row stride must be >= the row length");
    if (rows > 0 && cols > 0) {
        if (!p) return fail(CODED_ERR_ARG, what + " is NULL");
        if (!aligned(p, dt == CODED_F32 ? 4 : 2)) return fail(CODED_ERR_ARG, what + " is not aligned to its elements");
    }
    return CODED_OK;
}

}  // namespace
}  // namespace coded
