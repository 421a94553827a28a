// Microscaled matrices: what the host glue and the kernels share.
//
// Row t of a matrix holds blocks of 32 columns.  Block b has a scale byte B
// (value 2^(B - 127), 255: NaN) and 32 codes: E2M1, two a byte with the even
// column in the low bits, or E4M3, one a byte.  Codes start at 16-byte
// boundaries (row pitch a multiple of 16), scales at 4-byte ones.
#pragma once

#include "internal.h"

namespace coded {

constexpr int kMxBlock = 32;

struct MxMat {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t ldc, lds;   // bytes between rows
    int32_t bits;       // 4 or 8
};

// out (s right-hand sides) = alpha * product + beta * C.  The sum runs over
// `k` terms and there are `n` results for each right-hand side: mm sums along
// A's rows (k = r, n = q), mm_t across them (k = q, n = r).
struct MxArgs {
    MxMat A;
    MxMat XM;            // X, when it is microscaled too (x_bits != 0)
    const void* X;
    void* Y;
    const void* C;       // same type and order as Y, or null
    int64_t q, r, s;
    int64_t ldx, ldy, ldcc;
    float alpha, beta;
    int32_t x_bits;      // 0: X is dense
    int32_t x_bf16;      // dense X: bf16, else fp32
    int32_t y_bf16;
    int32_t x_rows;      // a right-hand side is a row of X
    int32_t y_rows;      // and of Y
    int32_t trans;
    void* workspace;
    int64_t workspace_bytes;
};

hipError_t launch_mx_quantize(const void* A, bool bf16, int64_t q, int64_t r, int64_t lda, const MxMat& out,
                              hipStream_t st);
hipError_t launch_mx_dequantize(const MxMat& m, int64_t q, int64_t r, void* out, bool bf16, int64_t ldo,
                                hipStream_t st);
hipError_t launch_mx_product(const MxArgs& a, hipStream_t st);
// Workspace bytes the product may use (0: none).
int64_t mx_workspace_bytes(const MxArgs& a);

// Few right-hand sides (mx_few.hip): whether it serves these sizes, and its parts of the two above.
bool mx_few_serves(const MxArgs& a);
int64_t mx_few_workspace_bytes(const MxArgs& a);
hipError_t launch_mx_few(const MxArgs& a, hipStream_t st);

// Many dense ones (mx_tiled.hip).
bool mx_tiled_serves(const MxArgs& a);
int64_t mx_tiled_workspace_bytes(const MxArgs& a);
hipError_t launch_mx_tiled(const MxArgs& a, hipStream_t st);
// Both sides in 4 bits (mx_scaled.hip).
bool mx_scaled_serves(const MxArgs& a);
int64_t mx_scaled_workspace_bytes(const MxArgs& a);
hipError_t launch_mx_scaled(const MxArgs& a, hipStream_t st);
// Y from partial sums part[split][side][result] of n results a side, added in order.
hipError_t launch_mx_join(const MxArgs& a, const float* part, int64_t splits, int64_t n, hipStream_t st);

#ifdef __HIPCC__
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));

// The scale 2^(B - 127) as the conversion instructions take it: they read the
// exponent field alone, and an exponent of 255 makes every result NaN.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two values of a code word, exact in bf16: codes 2 I and 2 I + 1 of 4 (8 bits)
// or 8 (4 bits).
template <int BITS, int I>
__device__ __forceinline__ uint32_t mx_pair_bf16(uint32_t word, float scale) {
    mx_bf16x2 v;
    if constexpr (BITS == 4)
        v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, I);
    else
        v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, I);
    return __builtin_bit_cast(uint32_t, v);
}
template <int BITS, int I>
__device__ __forceinline__ mx_f32x2 mx_pair_f32(uint32_t word, float scale) {
    if constexpr (BITS == 4)
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, I);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, scale, I);
}

// Eight consecutive values of one block as four words of bf16 pairs.  `at` is
// the first of the eight within the row (a multiple of 8).
template <int BITS>
__device__ __forceinline__ void mx_eight(const uint8_t* codes, const uint8_t* scales, int64_t at, uint32_t (&v)[4]) {
    const float s = mx_scale(scales[at / kMxBlock]);
    if constexpr (BITS == 4) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + at / 2);
        v[0] = mx_pair_bf16<4, 0>(w, s);
        v[1] = mx_pair_bf16<4, 1>(w, s);
        v[2] = mx_pair_bf16<4, 2>(w, s);
        v[3] = mx_pair_bf16<4, 3>(w, s);
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(codes + at);
        v[0] = mx_pair_bf16<8, 0>(w.x, s);
        v[1] = mx_pair_bf16<8, 1>(w.x, s);
        v[2] = mx_pair_bf16<8, 0>(w.y, s);
        v[3] = mx_pair_bf16<8, 1>(w.y, s);
    }
}

// An fp32 value as three bf16 values whose sum it is: its 24 significant bits,
// eight a piece, cut off and not rounded, so that no piece overflows.  An
// infinity or NaN is carried by the first piece alone.  (Pieces below 2^-133
// are lost: an absolute error of that size.)
__device__ __forceinline__ void split_bf16(float x, uint16_t (&p)[3]) {
    const uint32_t b = __float_as_uint(x);
    uint32_t hi = b & 0xFFFF0000u;
    if ((b & 0x7F800000u) == 0x7F800000u) {
        if (b & 0x007FFFFFu) hi |= 0x00400000u;   // a NaN whose payload lay in the bits cut off
        p[0] = hi >> 16;
        p[1] = p[2] = 0;
        return;
    }
    const float rest = x - __uint_as_float(hi);
    const uint32_t mid = __float_as_uint(rest) & 0xFFFF0000u;
    p[0] = hi >> 16;
    p[1] = mid >> 16;
    p[2] = __float_as_uint(rest - __uint_as_float(mid)) >> 16;
}

__device__ __forceinline__ uint16_t mx_to_bf16(float v) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));   // to nearest even
}

// One result: alpha * v + beta * C in fp32, rounded once.
__device__ __forceinline__ void mx_store(const MxArgs& a, int64_t side, int64_t j, float v) {
    const int64_t at = a.y_rows ? side * a.ldy + j : j * a.ldy + side;
    v *= a.alpha;
    if (a.C) {
        const int64_t ct = a.y_rows ? side * a.ldcc + j : j * a.ldcc + side;
        const float c = a.y_bf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.C)[ct]) << 16)
                                 : static_cast<const float*>(a.C)[ct];
        v = fmaf(a.beta, c, v);
    }
    if (a.y_bf16)
        static_cast<uint16_t*>(a.Y)[at] = mx_to_bf16(v);
    else
        static_cast<float*>(a.Y)[at] = v;
}
#endif

}  // namespace coded
