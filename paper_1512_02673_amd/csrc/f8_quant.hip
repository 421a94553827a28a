// 8-bit codes of a matrix and of its transpose, and back (the format of f8.h).
//
// A workgroup takes 128 x 128 values, which hold whole blocks whichever way they
// run: a thread 8 consecutive rows of 8 columns, in registers.  A row's maximum
// is taken over the 16 lanes that share it, a column's over a thread's rows, the
// wave and the four waves; 128 x 128 blocks take the largest of either.  Codes
// along rows are stored as they come, eight bytes a lane and 128 a row; those of
// the transpose change places in shared memory first, so that each of its rows
// is stored 16 bytes a lane and 128 a row too.
//
// With u = 448 / m rounded to fp32, v u is at most 448 (1 + 2^-23) and rounds to
// 448: no value has to be cut down.  m is 2^-100 at least, so u and m / 448 are
// normal numbers.
//
// Bound: memory.  Measured: 65536 x 8192 bf16 both ways 541 us (2.1 GB, 4.0 TB/s; a copy
// reaches 5.0: the transpose's rows take 128 bytes of every tile each), 16384 x 8192
// 147, 11500 x 5750 fp32 both ways 97 (4.1 TB/s); along rows alone 8192 x 8192 fp32 62
// (5.4 TB/s).  Back to bf16: 65536 x 8192 278 us (5.8 TB/s).
#include "f8.h"
#include "rows.h"

namespace coded {
namespace {

constexpr int kThreads = 256;
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The factor of a block's codes (0: a block without values) and its scale, from the bits of its largest magnitude.
__device__ __forceinline__ float factor_of(uint32_t m) {
    return m >= 0x7F800000u ? 0.0f : kF8Top / __uint_as_float(max(m, kF8Least));
}
__device__ __forceinline__ float scale_of(uint32_t m) {
    return m >= 0x7F800000u ? __builtin_nanf("") : __uint_as_float(max(m, kF8Least)) / kF8Top;
}

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// The code of v u; a block without values (u = 0) has codes of zero, whatever stands in it.
__device__ __forceinline__ float coded_value(float v, float u) { return u == 0.0f ? 0.0f : v * u; }

// ROWS, COLS: A's codes and its transpose's are written.
template <bool BF16, bool ROWS, bool COLS>
__global__ __launch_bounds__(kThreads) void f8_quantize_kernel(const void* A, int64_t q, int64_t r, int64_t lda, F8Mat m,
                                                              F8Mat t, int64_t tiles_c) {
    __shared__ uint32_t col_max[COLS ? 4 : 1][kF8Block];
    __shared__ uint32_t all_max[4];
    __shared__ __attribute__((aligned(16))) char turned[COLS ? kF8Block * kF8Block : 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 15, rg = tid >> 4;
    const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const int64_t r0 = tr * kF8Block + rg * 8, c0 = tc * kF8Block + cg * 8;
    float v[8][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (r0 + k < q) {
            row_load<BF16>(static_cast<const char*>(A) + (r0 + k) * lda * (BF16 ? 2 : 4), c0, r, v[k]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
        }
    }
    // magnitudes compare as their bits do, and infinities and NaN are the largest
    uint32_t row_max[8], own[8], most = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        row_max[k] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = magnitude(v[k][i]);
            row_max[k] = max(row_max[k], b);
            own[i] = k ? max(own[i], b) : b;
        }
        most = max(most, row_max[k]);
    }
    const bool all = (ROWS && m.block_rows != 1) || (COLS && t.block_rows != 1);
    if (ROWS && m.block_rows == 1) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int d = 1; d < 16; d *= 2) row_max[k] = max(row_max[k], static_cast<uint32_t>(__shfl_xor(static_cast<int>(row_max[k]), d)));
    }
    if (COLS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t x = own[i];
            x = max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), 16)));
            x = max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), 32)));
            if (lane < 16) col_max[wave][cg * 8 + i] = x;
        }
    }
    if (all) {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), d)));
        if (lane == 0) all_max[wave] = most;
    }
    if (COLS || all) __syncthreads();
    if (all) most = max(max(all_max[0], all_max[1]), max(all_max[2], all_max[3]));
    if constexpr (ROWS) {
        const bool whole = m.block_rows != 1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (r0 + k >= q) break;
            const uint32_t b = whole ? most : row_max[k];
            const float u = factor_of(b);
            uint2 w;
            w.x = four_codes(coded_value(v[k][0], u), coded_value(v[k][1], u), coded_value(v[k][2], u), coded_value(v[k][3], u));
            w.y = four_codes(coded_value(v[k][4], u), coded_value(v[k][5], u), coded_value(v[k][6], u), coded_value(v[k][7], u));
            *reinterpret_cast<uint2*>(m.codes + (r0 + k) * m.ldc + c0) = w;
            if (!whole && cg == 0) m.scales[tc * m.lds + r0 + k] = scale_of(b);
        }
        if (whole && tid == 0) m.scales[tc * m.lds + tr] = scale_of(most);
    }
    if constexpr (COLS) {
        const bool whole = t.block_rows != 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = cg * 8 + i;
            const uint32_t b = whole ? most : max(max(col_max[0][c], col_max[1][c]), max(col_max[2][c], col_max[3][c]));
            const float u = factor_of(b);
            uint2 w;
            w.x = four_codes(coded_value(v[0][i], u), coded_value(v[1][i], u), coded_value(v[2][i], u), coded_value(v[3][i], u));
            w.y = four_codes(coded_value(v[4][i], u), coded_value(v[5][i], u), coded_value(v[6][i], u), coded_value(v[7][i], u));
            *reinterpret_cast<uint2*>(turned + c * kF8Block + ((rg >> 1) ^ (cg & 7)) * 16 + (rg & 1) * 8) = w;
            if (!whole && rg == 0 && c0 + i < r) t.scales[tr * t.lds + c0 + i] = scale_of(b);
        }
        if (whole && tid == 0) t.scales[tr * t.lds + tc] = scale_of(most);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = k * 32 + (tid >> 3), piece = tid & 7;
            if (tc * kF8Block + c < r)
                *reinterpret_cast<u32x4_t*>(t.codes + (tc * kF8Block + c) * t.ldc + tr * kF8Block + piece * 16) =
                    *reinterpret_cast<const u32x4_t*>(turned + c * kF8Block + (piece ^ ((c >> 3) & 7)) * 16);
        }
    }
}

// A thread takes eight codes; short rows lie side by side in a workgroup, long ones are cut into pieces.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void f8_dequantize_kernel(F8Mat m, int64_t r, void* out, int64_t ldo, RowCut cut) {
    const int64_t row = blockIdx.x / cut.pieces * cut.rows(kThreads) + (threadIdx.x >> cut.log_tpr);
    const int64_t c0 = ((blockIdx.x % cut.pieces << cut.log_tpr) + (threadIdx.x & ((1 << cut.log_tpr) - 1))) * 8;
    if (row >= m.rows || c0 >= r) return;
    const uint2 w = *reinterpret_cast<const uint2*>(m.codes + row * m.ldc + c0);
    const float s = m.scales[c0 / kF8Block * m.lds + row / m.block_rows];
    mx_f32x2 v[4];
    v[0] = mx_pair_f32<8, 0>(w.x, 1.0f);
    v[1] = mx_pair_f32<8, 1>(w.x, 1.0f);
    v[2] = mx_pair_f32<8, 0>(w.y, 1.0f);
    v[3] = mx_pair_f32<8, 1>(w.y, 1.0f);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = v[i].x * s;
        f[2 * i + 1] = v[i].y * s;
    }
    row_store<BF16>(static_cast<char*>(out) + row * ldo * (BF16 ? 2 : 4), c0, r, f);
}

constexpr int64_t kMostBlocks = int64_t(1) << 23;   // half of what a grid takes

F8Mat from_row(F8Mat m, int64_t t) {   // t: a multiple of 128
    m.codes += t * m.ldc;
    m.scales += t / m.block_rows;
    m.rows -= t;
    return m;
}

template <bool BF16>
hipError_t quantize(const void* A, int64_t q, int64_t r, int64_t lda, const F8Mat* m, const F8Mat* t, hipStream_t st) {
    const int64_t tiles_c = ceil_div(r, kF8Block), step = kMostBlocks / tiles_c * kF8Block;
    if (step < 1) return hipErrorInvalidConfiguration;
    const auto kernel = m && t ? f8_quantize_kernel<BF16, true, true> : m ? f8_quantize_kernel<BF16, true, false> : f8_quantize_kernel<BF16, false, true>;
    for (int64_t at = 0; at < q; at += step) {
        const int64_t rows = lesser(step, q - at);
        F8Mat tt = t ? *t : F8Mat{};
        if (t) {   // its columns from `at` on
            tt.codes += at;
            tt.scales += at / kF8Block * tt.lds;
        }
        kernel<<<dim3(static_cast<uint32_t>(ceil_div(rows, kF8Block) * tiles_c)), kThreads, 0, st>>>(
            static_cast<const char*>(A) + at * lda * (BF16 ? 2 : 4), rows, r, lda, m ? from_row(*m, at) : F8Mat{}, tt, tiles_c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_f8_quantize(const void* A, bool bf16, int64_t q, int64_t r, int64_t lda, const F8Mat* m,
                              const F8Mat* t, hipStream_t st) {
    return bf16 ? quantize<true>(A, q, r, lda, m, t, st) : quantize<false>(A, q, r, lda, m, t, st);
}

hipError_t launch_f8_dequantize(const F8Mat& m, int64_t r, void* out, bool bf16, int64_t ldo, hipStream_t st) {
    const RowCut cut = cut_rows(r, 8);
    const int64_t step = kMostBlocks / cut.pieces * cut.rows(kThreads) / kF8Block * kF8Block;   // rows of a launch
    if (step < 1) return hipErrorInvalidConfiguration;
    for (int64_t at = 0; at < m.rows; at += step) {
        F8Mat part = from_row(m, at);
        part.rows = lesser(step, part.rows);
        const dim3 grid(static_cast<uint32_t>(ceil_div(part.rows, cut.rows(kThreads)) * cut.pieces));
        void* o = static_cast<char*>(out) + at * ldo * (bf16 ? 2 : 4);
        const auto kernel = bf16 ? f8_dequantize_kernel<true> : f8_dequantize_kernel<false>;
        kernel<<<grid, kThreads, 0, st>>>(part, r, o, ldo, cut);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace coded
