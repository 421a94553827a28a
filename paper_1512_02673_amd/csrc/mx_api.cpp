// C ABI of the microscaled matrices: argument checks, then the launches.
#include <algorithm>
#include <cmath>
#include <limits>

#include "api_checks.h"
#include "mx.h"

namespace coded {
namespace {

int bits_of(coded_dtype fmt) { return fmt == CODED_MX4 ? 4 : fmt == CODED_MX8 ? 8 : 0; }

int64_t code_pitch(int bits, int64_t r) { return ceil_div(r, kMxBlock) * kMxBlock / 8 * bits; }
int64_t scale_pitch(int64_t r) { return ceil_div(ceil_div(r, kMxBlock), 4) * 4; }

// What every call asks of a microscaled rows x cols operand.
coded_status check_mx(const char* name, coded_dtype fmt, const void* codes, int64_t ldc, const uint8_t* scales, int64_t lds,
                      int64_t rows, int64_t cols, MxMat& out) {
    const std::string what(name);
    const int bits = bits_of(fmt);
    if (!bits) return fail(CODED_ERR_ARG, what + ": the format must be CODED_MX4 or CODED_MX8");
    if (rows < 0 || cols < 0) return fail(CODED_ERR_SHAPE, what + ": sizes must be >= 0");
    if (cols > kMostSize || rows > kMostSize) return fail(CODED_ERR_SHAPE, what + ": sizes must be <= 2^40");
    if (ldc < code_pitch(bits, cols) || ldc % 16 != 0)
        return fail(CODED_ERR_SHAPE, what + ": the code pitch must be a multiple of 16 bytes that holds a row");
    if (lds < scale_pitch(cols) || lds % 4 != 0)
        return fail(CODED_ERR_SHAPE, what + ": the scale pitch must be a multiple of 4 bytes that holds a row");
    if (rows > 0 && cols > 0) {
        if (!codes || !scales) return fail(CODED_ERR_ARG, what + ": codes or scales is NULL");
        if (!aligned(codes, 16)) return fail(CODED_ERR_ARG, what + ": codes must be 16-byte aligned");
        if (!aligned(scales, 4)) return fail(CODED_ERR_ARG, what + ": scales must be 4-byte aligned");
    }
    out = MxMat{static_cast<const uint8_t*>(codes), scales, ldc, lds, bits};
    return CODED_OK;
}

coded_status product(bool trans, coded_dtype fmt, const void* codes, int64_t ldc, const uint8_t* scales, int64_t lds,
                     int64_t q, int64_t r, coded_dtype x_dt, const void* X, int64_t ldx, const uint8_t* x_scales,
                     int64_t ldxs, int64_t s, int32_t order, double alpha, double beta, const void* C, int64_t ldcc,
                     void* Y, coded_dtype y_dt, int64_t ldy, void* workspace, int64_t workspace_bytes, void* stream) {
    MxArgs a{};
    coded_status st = check_mx("A", fmt, codes, ldc, scales, lds, q, r, a.A);
    if (st != CODED_OK) return st;
    if (s < 0 || s > kMostSize) return fail(CODED_ERR_SHAPE, "s must be in [0, 2^40]");
    if (order & ~(CODED_X_ROWS | CODED_Y_ROWS)) return fail(CODED_ERR_ARG, "order has unknown bits");
    a.q = q;
    a.r = r;
    a.s = s;
    a.trans = trans;
    a.x_rows = (order & CODED_X_ROWS) != 0;
    a.y_rows = (order & CODED_Y_ROWS) != 0;
    const int64_t k = trans ? q : r, n = trans ? r : q;
    if (!trans && bits_of(x_dt)) {
        if (!a.x_rows) return fail(CODED_ERR_UNSUPPORTED, "a microscaled X holds a right-hand side a row (CODED_X_ROWS)");
        st = check_mx("X", x_dt, X, ldx, x_scales, ldxs, s, k, a.XM);
        a.x_bits = a.XM.bits;
    } else {
        st = a.x_rows ? check_dense("X", x_dt, X, s, k, ldx) : check_dense("X", x_dt, X, k, s, ldx);
        a.X = X;
        a.ldx = ldx;
        a.x_bf16 = x_dt == CODED_BF16;
    }
    if (st != CODED_OK) return st;
    const int64_t rows = a.y_rows ? s : n, cols = a.y_rows ? n : s;
    st = check_dense("Y", y_dt, Y, rows, cols, ldy);
    if (st != CODED_OK) return st;
    const double top = std::numeric_limits<float>::max();   // they enter in fp32
    if (!(std::fabs(alpha) <= top && std::fabs(beta) <= top)) return fail(CODED_ERR_ARG, "alpha and beta must be finite in fp32");
    a.alpha = static_cast<float>(alpha);
    a.beta = static_cast<float>(beta);
    if (beta != 0.0) {
        // a row stride of 0 gives every row of Y the same row of C
        st = check_dense("C", y_dt, C, rows, cols, ldcc == 0 ? std::max<int64_t>(cols, 1) : ldcc);
        if (st != CODED_OK) return st;
        if (ldcc == 0 && C == Y && rows > 1) return fail(CODED_ERR_ARG, "a C of one row for every row of Y must not be Y");
        a.C = C;
        a.ldcc = ldcc;
    }
    a.Y = Y;
    a.ldy = ldy;
    a.y_bf16 = y_dt == CODED_BF16;
    if (n == 0 || s == 0) return CODED_OK;
    const int64_t need = mx_workspace_bytes(a);
    if (need > 0) {
        if (!workspace || workspace_bytes < need)
            return fail(CODED_ERR_ARG, "the workspace must have " + std::to_string(need) + " bytes");
        if (!aligned(workspace, 16)) return fail(CODED_ERR_ARG, "the workspace must be 16-byte aligned");
    }
    a.workspace = workspace;
    a.workspace_bytes = workspace_bytes;
    const hipError_t e = launch_mx_product(a, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? CODED_OK : hip_fail(e, trans ? "coded_mx_mm_t" : "coded_mx_mm");
}

}  // namespace
}  // namespace coded

using namespace coded;

extern "C" {

coded_status coded_mx_sizes(coded_dtype fmt, int64_t r, int64_t* code_pitch_out, int64_t* scale_pitch_out) {
    return guarded([&] {
        const int bits = bits_of(fmt);
        if (!bits) return fail(CODED_ERR_ARG, "the format must be CODED_MX4 or CODED_MX8");
        if (r < 0 || r > kMostSize) return fail(CODED_ERR_SHAPE, "r must be in [0, 2^40]");
        if (code_pitch_out) *code_pitch_out = code_pitch(bits, r);
        if (scale_pitch_out) *scale_pitch_out = scale_pitch(r);
        return CODED_OK;
    });
}

coded_status coded_mx_workspace(int32_t transposed, coded_dtype fmt, int64_t q, int64_t r, coded_dtype x_dt, int64_t s,
                                int32_t order, int64_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(CODED_ERR_ARG, "bytes is NULL");
        if (!bits_of(fmt)) return fail(CODED_ERR_ARG, "the format must be CODED_MX4 or CODED_MX8");
        if (x_dt != CODED_F32 && x_dt != CODED_BF16 && (transposed || !bits_of(x_dt)))
            return fail(CODED_ERR_ARG, "x_dt is not a type of X");
        if (q < 0 || r < 0 || s < 0 || std::max(std::max(q, r), s) > kMostSize) return fail(CODED_ERR_SHAPE, "sizes must be in [0, 2^40]");
        if (order & ~(CODED_X_ROWS | CODED_Y_ROWS)) return fail(CODED_ERR_ARG, "order has unknown bits");
        MxArgs a{};
        a.A.bits = bits_of(fmt);
        a.q = q;
        a.r = r;
        a.s = s;
        a.trans = transposed != 0;
        a.x_bits = bits_of(x_dt);
        a.x_bf16 = x_dt == CODED_BF16;
        a.x_rows = (order & CODED_X_ROWS) != 0;
        a.y_rows = (order & CODED_Y_ROWS) != 0;
        *bytes = (transposed ? r : q) == 0 || s == 0 ? 0 : mx_workspace_bytes(a);
        return CODED_OK;
    });
}

coded_status coded_mx_quantize(coded_dtype dt, const void* A, int64_t q, int64_t r, int64_t lda, coded_dtype fmt,
                               void* codes, int64_t ldc, uint8_t* scales, int64_t lds, void* stream) {
    return guarded([&] {
        MxMat m{};
        coded_status st = check_mx("M", fmt, codes, ldc, scales, lds, q, r, m);
        if (st == CODED_OK) st = check_dense("A", dt, A, q, r, lda);
        if (st != CODED_OK) return st;
        if (q == 0 || r == 0) return CODED_OK;
        const hipError_t e = launch_mx_quantize(A, dt == CODED_BF16, q, r, lda, m, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_mx_quantize");
    });
}

coded_status coded_mx_dequantize(coded_dtype fmt, const void* codes, int64_t ldc, const uint8_t* scales, int64_t lds,
                                 int64_t q, int64_t r, coded_dtype dt, void* out, int64_t ldo, void* stream) {
    return guarded([&] {
        MxMat m{};
        coded_status st = check_mx("M", fmt, codes, ldc, scales, lds, q, r, m);
        if (st == CODED_OK) st = check_dense("out", dt, out, q, r, ldo);
        if (st != CODED_OK) return st;
        if (q == 0 || r == 0) return CODED_OK;
        const hipError_t e = launch_mx_dequantize(m, q, r, out, dt == CODED_BF16, ldo, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_mx_dequantize");
    });
}

coded_status coded_mx_mm(coded_dtype fmt, const void* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t q,
                         int64_t r, coded_dtype x_dt, const void* X, int64_t ldx, const uint8_t* x_scales, int64_t ldxs,
                         int64_t s, int32_t order, double alpha, double beta, const void* C, int64_t ldcc, void* Y,
                         coded_dtype y_dt, int64_t ldy, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] {
        return product(false, fmt, codes, ldc, scales, lds, q, r, x_dt, X, ldx, x_scales, ldxs, s, order, alpha, beta, C,
                       ldcc, Y, y_dt, ldy, workspace, workspace_bytes, stream);
    });
}

coded_status coded_mx_mm_t(coded_dtype fmt, const void* codes, int64_t ldc, const uint8_t* scales, int64_t lds,
                           int64_t q, int64_t r, coded_dtype u_dt, const void* U, int64_t ldu, int64_t s, int32_t order,
                           double alpha, double beta, const void* C, int64_t ldcc, void* Z, coded_dtype z_dt,
                           int64_t ldz, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] {
        return product(true, fmt, codes, ldc, scales, lds, q, r, u_dt, U, ldu, nullptr, 0, s, order, alpha, beta, C, ldcc,
                       Z, z_dt, ldz, workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
