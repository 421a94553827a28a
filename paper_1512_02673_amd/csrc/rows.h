// Rows of fp32 or bf16, eight elements a thread, at any element's boundary.
#pragma once

#include "mx_window.h"

namespace coded {
namespace {

#ifdef __HIPCC__
typedef u32x4_t u32x4_bf __attribute__((aligned(2)));   // 16 bytes at any bf16 boundary
typedef u32x4_t u32x4_f __attribute__((aligned(4)));    // 16 bytes at any fp32 boundary

// Eight elements of a row from column c on, as many as there are: v[i] for c + i < cols, the others zero.
template <bool BF16>
__device__ __forceinline__ void row_load(const void* row, int64_t c, int64_t cols, float (&v)[8]) {
    if (c + 8 <= cols) {
        if constexpr (BF16) {
            const u32x4_t w = *reinterpret_cast<const u32x4_bf*>(static_cast<const uint16_t*>(row) + c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const u32x4_f* p = reinterpret_cast<const u32x4_f*>(static_cast<const float*>(row) + c);
            const u32x4_t lo = p[0], hi = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = __uint_as_float(lo[i]);
                v[4 + i] = __uint_as_float(hi[i]);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        if (c + i < cols) {
            if constexpr (BF16)
                v[i] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[c + i]) << 16);
            else
                v[i] = static_cast<const float*>(row)[c + i];
        }
    }
}
template <bool BF16>
__device__ __forceinline__ void row_store(void* row, int64_t c, int64_t cols, const float (&v)[8]) {
    if constexpr (BF16) {
        uint16_t* o = static_cast<uint16_t*>(row) + c;
        u32x4_t p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = mx_to_bf16(v[2 * i]) | static_cast<uint32_t>(mx_to_bf16(v[2 * i + 1])) << 16;
        if (c + 8 <= cols) {
            *reinterpret_cast<u32x4_bf*>(o) = p;
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (c + i < cols) o[i] = static_cast<uint16_t>(p[i / 2] >> (16 * (i & 1)));
    } else {
        float* o = static_cast<float*>(row) + c;
        if (c + 8 <= cols) {
            reinterpret_cast<u32x4_f*>(o)[0] = u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            reinterpret_cast<u32x4_f*>(o)[1] = u32x4_t{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (c + i < cols) o[i] = v[i];
    }
}
#endif

// Threads on a row (a power of two up to `threads`, eight columns each) and pieces of a row.
struct RowCut {
    int log_tpr;
    int64_t pieces;
    __host__ __device__ int rows(int threads) const { return threads >> log_tpr; }
};
inline RowCut cut_rows(int64_t cols, int log_threads) {
    const int64_t want = ceil_div(cols, 8);
    int l = 0;
    while (l < log_threads && (int64_t(1) << l) < want) ++l;
    return {l, ceil_div(want, int64_t(1) << l)};
}

}  // namespace
}  // namespace coded
