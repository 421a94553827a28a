// C ABI of the matrices in 8 bits with blocks of 128: argument checks, then the launches.
#include <algorithm>
#include <cmath>
#include <limits>

#include "api_checks.h"
#include "f8.h"

namespace coded {
namespace {

constexpr int64_t kMostTerms = int64_t(1) << 23, kMostPitch = int64_t(1) << 24;   // of a product
constexpr int64_t kMostStored = int64_t(1) << 27;                                  // columns of a matrix that is stored or read back

int64_t code_pitch(int64_t r) { return ceil_div(r, kF8Block) * kF8Block; }

// What every call asks of a rows x cols operand.
coded_status check_f8(const char* name, int32_t block_rows, const void* codes, int64_t ldc, const float* scales, int64_t lds,
                      int64_t rows, int64_t cols, F8Mat& out) {
    const std::string what(name);
    if (block_rows != 1 && block_rows != kF8Block) return fail(CODED_ERR_ARG, what + ": a block must have 1 or 128 rows");
    if (rows < 0 || cols < 0) return fail(CODED_ERR_SHAPE, what + ": sizes must be >= 0");
    if (cols > kMostSize || rows > kMostSize) return fail(CODED_ERR_SHAPE, what + ": sizes must be <= 2^40");
    if (ldc < code_pitch(cols) || ldc % 16 != 0)
        return fail(CODED_ERR_SHAPE, what + ": the code pitch must be a multiple of 16 bytes that holds a row's blocks");
    if (lds < ceil_div(rows, block_rows)) return fail(CODED_ERR_SHAPE, what + ": the scale pitch must hold the rows' blocks");
    if (rows > 0 && cols > 0) {
        if (!codes || !scales) return fail(CODED_ERR_ARG, what + ": codes or scales is NULL");
        if (!aligned(codes, 16)) return fail(CODED_ERR_ARG, what + ": codes must be 16-byte aligned");
        if (!aligned(scales, 4)) return fail(CODED_ERR_ARG, what + ": scales must be 4-byte aligned");
    }
    out = F8Mat{static_cast<uint8_t*>(const_cast<void*>(codes)), const_cast<float*>(scales), ldc, lds, rows, block_rows};
    return CODED_OK;
}

// Y holds results of X's rows for A's (q x s) or, with y_rows, the other way round.
void set_sides(F8Args& a, const F8Mat& A, const F8Mat& X, int64_t q, int64_t r, int64_t s, bool y_rows) {
    a.P = X;
    a.Q = A;
    a.o.q = q;
    a.o.r = r;
    a.o.s = s;
    a.o.y_rows = y_rows;
    a.blocks = ceil_div(r, kF8Block);
}

}  // namespace
}  // namespace coded

using namespace coded;

extern "C" {

coded_status coded_f8_sizes(int64_t q, int64_t r, int32_t block_rows, int64_t* code_pitch_out, int64_t* scale_pitch_out) {
    return guarded([&] {
        if (block_rows != 1 && block_rows != kF8Block) return fail(CODED_ERR_ARG, "a block must have 1 or 128 rows");
        if (q < 0 || r < 0 || std::max(q, r) > kMostSize) return fail(CODED_ERR_SHAPE, "sizes must be in [0, 2^40]");
        if (code_pitch_out) *code_pitch_out = code_pitch(r);
        if (scale_pitch_out) *scale_pitch_out = ceil_div(q, block_rows);
        return CODED_OK;
    });
}

coded_status coded_f8_quantize(coded_dtype dt, const void* A, int64_t q, int64_t r, int64_t lda, int32_t block_rows,
                               void* codes, int64_t ldc, float* scales, int64_t lds, int32_t t_block_rows,
                               void* t_codes, int64_t ldtc, float* t_scales, int64_t ldts, void* stream) {
    return guarded([&] {
        const bool rows = codes || scales, cols = t_codes || t_scales;
        if (q < 0 || r < 0 || std::max(q, r) > kMostSize) return fail(CODED_ERR_SHAPE, "sizes must be in [0, 2^40]");
        coded_status st = check_dense("A", dt, A, q, r, lda);
        F8Mat m{}, t{};
        if (st == CODED_OK && rows) st = check_f8("M", block_rows, codes, ldc, scales, lds, q, r, m);
        if (st == CODED_OK && cols) st = check_f8("MT", t_block_rows, t_codes, ldtc, t_scales, ldts, r, q, t);
        if (st != CODED_OK) return st;
        if (q == 0 || r == 0) return CODED_OK;
        if (r > kMostStored) return fail(CODED_ERR_UNSUPPORTED, "r must be <= 2^27");
        if (!rows && !cols) return fail(CODED_ERR_ARG, "neither A's codes nor its transpose's are given");
        const hipError_t e = launch_f8_quantize(A, dt == CODED_BF16, q, r, lda, rows ? &m : nullptr, cols ? &t : nullptr,
                                                static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_f8_quantize");
    });
}

coded_status coded_f8_dequantize(int64_t q, int64_t r, int32_t block_rows, const void* codes, int64_t ldc,
                                 const float* scales, int64_t lds, coded_dtype dt, void* out, int64_t ldo, void* stream) {
    return guarded([&] {
        F8Mat m{};
        coded_status st = check_f8("M", block_rows, codes, ldc, scales, lds, q, r, m);
        if (st == CODED_OK) st = check_dense("out", dt, out, q, r, ldo);
        if (st != CODED_OK) return st;
        if (q == 0 || r == 0) return CODED_OK;
        if (r > kMostStored) return fail(CODED_ERR_UNSUPPORTED, "r must be <= 2^27");
        const hipError_t e = launch_f8_dequantize(m, r, out, dt == CODED_BF16, ldo, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_f8_dequantize");
    });
}

coded_status coded_f8_workspace(int64_t q, int64_t r, int64_t s, coded_dtype y_dt, int32_t order, int64_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(CODED_ERR_ARG, "bytes is NULL");
        if (q < 0 || r < 0 || s < 0 || std::max(std::max(q, r), s) > kMostSize) return fail(CODED_ERR_SHAPE, "sizes must be in [0, 2^40]");
        if (r > kMostTerms) return fail(CODED_ERR_UNSUPPORTED, "r must be <= 2^23");
        if (y_dt != CODED_F32 && y_dt != CODED_BF16) return fail(CODED_ERR_ARG, "Y must be CODED_F32 or CODED_BF16");
        if (order & ~CODED_Y_ROWS) return fail(CODED_ERR_ARG, "order has unknown bits");
        F8Args a{};
        set_sides(a, F8Mat{}, F8Mat{}, q, r, s, (order & CODED_Y_ROWS) != 0);
        a.o.y_bf16 = y_dt == CODED_BF16;
        *bytes = q == 0 || s == 0 ? 0 : f8_workspace_bytes(a);
        return CODED_OK;
    });
}

coded_status coded_f8_mm(int64_t q, int64_t r, int64_t s, int32_t block_rows, const void* codes, int64_t ldc,
                         const float* scales, int64_t lds, int32_t x_block_rows, const void* x_codes, int64_t ldxc,
                         const float* x_scales, int64_t ldxs, int32_t order, double alpha, double beta, const void* C,
                         int64_t ldcc, void* Y, coded_dtype y_dt, int64_t ldy, void* workspace, int64_t workspace_bytes,
                         void* stream) {
    return guarded([&] {
        F8Mat A{}, X{};
        coded_status st = check_f8("A", block_rows, codes, ldc, scales, lds, q, r, A);
        if (st == CODED_OK) st = check_f8("X", x_block_rows, x_codes, ldxc, x_scales, ldxs, s, r, X);
        if (st != CODED_OK) return st;
        if (order & ~CODED_Y_ROWS) return fail(CODED_ERR_ARG, "order has unknown bits");
        F8Args a{};
        set_sides(a, A, X, q, r, s, (order & CODED_Y_ROWS) != 0);
        const int64_t rows = a.o.y_rows ? s : q, cols = a.o.y_rows ? q : s;
        st = check_dense("Y", y_dt, Y, rows, cols, ldy);
        if (st != CODED_OK) return st;
        const double top = std::numeric_limits<float>::max();   // they enter in fp32
        if (!(std::fabs(alpha) <= top && std::fabs(beta) <= top)) return fail(CODED_ERR_ARG, "alpha and beta must be finite in fp32");
        a.o.alpha = static_cast<float>(alpha);
        a.o.beta = static_cast<float>(beta);
        if (beta != 0.0) {
            // a row stride of 0 gives every row of Y the same row of C
            st = check_dense("C", y_dt, C, rows, cols, ldcc == 0 ? std::max<int64_t>(cols, 1) : ldcc);
            if (st != CODED_OK) return st;
            if (ldcc == 0 && C == Y && rows > 1) return fail(CODED_ERR_ARG, "a C of one row for every row of Y must not be Y");
            a.o.C = C;
            a.o.ldcc = ldcc;
        }
        a.o.Y = Y;
        a.o.ldy = ldy;
        a.o.y_bf16 = y_dt == CODED_BF16;
        if (r > kMostTerms) return fail(CODED_ERR_UNSUPPORTED, "r must be <= 2^23");
        if (std::max(ldc, ldxc) > kMostPitch) return fail(CODED_ERR_UNSUPPORTED, "code pitches must be <= 2^24");
        if (q == 0 || s == 0) return CODED_OK;
        const int64_t need = f8_workspace_bytes(a);
        if (need > 0) {
            if (!workspace || workspace_bytes < need)
                return fail(CODED_ERR_ARG, "the workspace must have " + std::to_string(need) + " bytes");
            if (!aligned(workspace, 16)) return fail(CODED_ERR_ARG, "the workspace must be 16-byte aligned");
        }
        a.o.workspace = workspace;
        a.o.workspace_bytes = workspace_bytes;
        const hipError_t e = launch_f8_product(a, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_f8_mm");
    });
}

}  // extern "C"
