// Microscaled codes of a matrix, and back (the block format of mx.h).
//
// m = max |v| of a block; the scale is 2^e with e = floor(log2 m) - emax, emax
// = 2 (E2M1) or 8 (E4M3) the exponent of the format's largest value, and at
// least -117: below that a value is under 2^-108 at most and its codes' values
// would leave bf16's normal range.  Codes are v / 2^e to nearest, ties to even,
// at most the format's largest value (a maximum between it and the next power
// of two is cut down to it).  A block with an infinity or NaN in it gets the
// NaN scale: all its values read back as NaN, and nothing hides the loss.
//
// Bound: memory.  Measured: 65536 x 8192 bf16 to 8 bits 330 to 350 us (1.62 GB, 4.6 to
// 4.9 TB/s; a copy reaches 4.7) and back 280 to 295 (5.5 TB/s), 11500 x 5750 fp32 to 4
// bits 61 us (4.9 TB/s) and back to bf16 26 (6.4).  Non-temporal loads and stores
// were no faster.
#include "mx.h"

namespace coded {
namespace {

constexpr int kThreads = 256;
constexpr int kMinScale = 10;   // 2^-117
constexpr uint32_t kNanScale = 255;

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t u32x4_bf __attribute__((aligned(2)));   // 16 bytes at any bf16 boundary
typedef u32x4_t u32x4_f __attribute__((aligned(4)));    // 16 bytes at any fp32 boundary
typedef short s16x2_t __attribute__((ext_vector_type(2)));

// A thread takes eight values, so four consecutive lanes share a block: its
// maximum takes two exchanges within the quad.  A wave reads 64 * 8 consecutive
// values of a row; a workgroup takes `rows` short rows or a piece of a long one.
template <int BITS, bool BF16>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const void* A, int64_t q, int64_t r, int64_t lda,
                                                              MxMat out, int log_tpr, int64_t pieces) {
    const int tpr = 1 << log_tpr;   // threads on a row: a multiple of 4
    const int64_t row = blockIdx.x / pieces * (kThreads >> log_tpr) + (threadIdx.x >> log_tpr);
    const int64_t c0 = ((blockIdx.x % pieces) * tpr + (threadIdx.x & (tpr - 1))) * 8;
    if (row >= q) return;   // whole quads leave together
    float v[8];
    if (c0 + 8 <= r) {
        if constexpr (BF16) {
            const u32x4_t w = *reinterpret_cast<const u32x4_bf*>(static_cast<const uint16_t*>(A) + row * lda + c0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        } else {
            const u32x4_f* p = reinterpret_cast<const u32x4_f*>(static_cast<const float*>(A) + row * lda + c0);
            const u32x4_t lo = p[0], hi = p[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = __uint_as_float(lo[i]);
                v[4 + i] = __uint_as_float(hi[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.0f;
            if (c0 + i < r) {
                if constexpr (BF16)
                    v[i] = __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(A)[row * lda + c0 + i])
                                           << 16);
                else
                    v[i] = static_cast<const float*>(A)[row * lda + c0 + i];
            }
        }
    }
    // magnitudes compare as their bits do, and infinities and NaN are the largest
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(m), 0xB1, 0xF, 0xF, true)));   // lane ^ 1
    m = max(m, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(m), 0x4E, 0xF, 0xF, true)));   // lane ^ 2
    const int biased = static_cast<int>(m >> 23);
    const bool fine = biased != 255;
    const uint32_t byte = fine ? static_cast<uint32_t>(max(biased - (BITS == 4 ? 2 : 8), kMinScale)) : kNanScale;
    const float s = mx_scale(fine ? byte : 127u);
    if (c0 >= (r + kMxBlock - 1) / kMxBlock * kMxBlock) {
        // past the last block: the scale bytes up to the next multiple of four are zero
        if ((threadIdx.x & 3) == 0 && c0 < (r + 127) / 128 * 128)
            const_cast<uint8_t*>(out.scales)[row * out.lds + c0 / kMxBlock] = 0;
        return;
    }
    if constexpr (BITS == 4) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
        *reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(out.codes) + row * out.ldc + c0 / 2) = fine ? w : 0u;
    } else {
        // the conversion makes NaN of what rounds past 448
        const float top = 448.0f * s;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fminf(fmaxf(v[i], -top), top);
        s16x2_t lo = {0, 0}, hi = {0, 0};
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[0], v[1], s, false);
        lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, v[2], v[3], s, true);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[4], v[5], s, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(hi, v[6], v[7], s, true);
        uint2 w = {__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
        if (!fine) w = {0u, 0u};
        *reinterpret_cast<uint2*>(const_cast<uint8_t*>(out.codes) + row * out.ldc + c0) = w;
    }
    if ((threadIdx.x & 3) == 0) const_cast<uint8_t*>(out.scales)[row * out.lds + c0 / kMxBlock] = byte;
}

// Same split: a thread writes eight values.
template <int BITS, bool BF16>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(MxMat m, int64_t q, int64_t r, void* out, int64_t ldo,
                                                                int log_tpr, int64_t pieces) {
    const int tpr = 1 << log_tpr;
    const int64_t row = blockIdx.x / pieces * (kThreads >> log_tpr) + (threadIdx.x >> log_tpr);
    const int64_t c0 = ((blockIdx.x % pieces) * tpr + (threadIdx.x & (tpr - 1))) * 8;
    if (row >= q || c0 >= r) return;
    const uint8_t* codes = m.codes + row * m.ldc;
    const float s = mx_scale(m.scales[row * m.lds + c0 / kMxBlock]);
    mx_f32x2 v[4];
    if constexpr (BITS == 4) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + c0 / 2);
        v[0] = mx_pair_f32<4, 0>(w, s);
        v[1] = mx_pair_f32<4, 1>(w, s);
        v[2] = mx_pair_f32<4, 2>(w, s);
        v[3] = mx_pair_f32<4, 3>(w, s);
    } else {
        const uint2 w = *reinterpret_cast<const uint2*>(codes + c0);
        v[0] = mx_pair_f32<8, 0>(w.x, s);
        v[1] = mx_pair_f32<8, 1>(w.x, s);
        v[2] = mx_pair_f32<8, 0>(w.y, s);
        v[3] = mx_pair_f32<8, 1>(w.y, s);
    }
    if constexpr (BF16) {
        u32x4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i)   // to nearest: exact for every scale from 2^-117
            w[i] = mx_to_bf16(v[i].x) | static_cast<uint32_t>(mx_to_bf16(v[i].y)) << 16;
        uint16_t* o = static_cast<uint16_t*>(out) + row * ldo + c0;
        if (c0 + 8 <= r) {
            *reinterpret_cast<u32x4_bf*>(o) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (c0 + i < r) o[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i & 1)));
        }
    } else {
        float* o = static_cast<float*>(out) + row * ldo + c0;
        if (c0 + 8 <= r) {
            reinterpret_cast<u32x4_f*>(o)[0] = u32x4_t{__float_as_uint(v[0].x), __float_as_uint(v[0].y),
                                                       __float_as_uint(v[1].x), __float_as_uint(v[1].y)};
            reinterpret_cast<u32x4_f*>(o)[1] = u32x4_t{__float_as_uint(v[2].x), __float_as_uint(v[2].y),
                                                       __float_as_uint(v[3].x), __float_as_uint(v[3].y)};
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (c0 + i < r) o[i] = i & 1 ? v[i / 2].y : v[i / 2].x;
        }
    }
}

// Threads on a row (a power of two from 4 to the workgroup), pieces of a row, rows a launch takes.
struct RowSplit {
    int log_tpr;
    int64_t pieces, rows;
    int64_t blocks(int64_t q) const { return ceil_div(q, kThreads >> log_tpr) * pieces; }
};
RowSplit split_rows(int64_t cols) {
    const int64_t want = ceil_div(cols, 8);
    int l = 2;
    while (l < 8 && (int64_t(1) << l) < want) ++l;
    const int64_t pieces = ceil_div(want, int64_t(1) << l);
    return {l, pieces, (int64_t(1) << 23) / pieces * (kThreads >> l)};   // half of what a grid takes
}

// f(first row, rows, blocks, split) for as many launches as the rows need.
template <class F>
hipError_t over_rows(int64_t q, int64_t cols, F f) {
    const RowSplit w = split_rows(cols);
    if (w.rows < 1) return hipErrorInvalidConfiguration;
    for (int64_t t = 0; t < q; t += w.rows) {
        const int64_t rows = q - t < w.rows ? q - t : w.rows;
        f(t, rows, dim3(static_cast<uint32_t>(w.blocks(rows))), w);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

MxMat from_row(MxMat m, int64_t t) {
    m.codes += t * m.ldc;
    m.scales += t * m.lds;
    return m;
}

}  // namespace

hipError_t launch_mx_quantize(const void* A, bool bf16, int64_t q, int64_t r, int64_t lda, const MxMat& out,
                              hipStream_t st) {
    // columns up to the end of the scales' last word
    return over_rows(q, ceil_div(r, 128) * 128, [&](int64_t t, int64_t rows, dim3 grid, const RowSplit& w) {
        const void* a = static_cast<const char*>(A) + t * lda * (bf16 ? 2 : 4);
        const MxMat o = from_row(out, t);
        const auto kernel = o.bits == 4 ? (bf16 ? mx_quantize_kernel<4, true> : mx_quantize_kernel<4, false>)
                                        : (bf16 ? mx_quantize_kernel<8, true> : mx_quantize_kernel<8, false>);
        kernel<<<grid, kThreads, 0, st>>>(a, rows, r, lda, o, w.log_tpr, w.pieces);
    });
}

hipError_t launch_mx_dequantize(const MxMat& m, int64_t q, int64_t r, void* out, bool bf16, int64_t ldo,
                                hipStream_t st) {
    return over_rows(q, r, [&](int64_t t, int64_t rows, dim3 grid, const RowSplit& w) {
        void* o = static_cast<char*>(out) + t * ldo * (bf16 ? 2 : 4);
        const auto kernel = m.bits == 4 ? (bf16 ? mx_dequantize_kernel<4, true> : mx_dequantize_kernel<4, false>)
                                        : (bf16 ? mx_dequantize_kernel<8, true> : mx_dequantize_kernel<8, false>);
        kernel<<<grid, kThreads, 0, st>>>(from_row(m, t), rows, r, o, ldo, w.log_tpr, w.pieces);
    });
}

}  // namespace coded
