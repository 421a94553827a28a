// C ABI of dropout and embeddings: argument checks, then the launches.
#include <cmath>
#include <limits>

#include "api_checks.h"
#include "layers.h"

using namespace coded;

namespace {

constexpr uint64_t kDropoutStream = 10;   // of the seed's generator
constexpr double kTop = std::numeric_limits<float>::max();

constexpr int64_t kMostColumns = int64_t(1) << 33;

coded_status check_sizes(int64_t rows, int64_t columns) {
    if (rows < 0 || columns < 0 || std::max(rows, columns) > kMostSize) return fail(CODED_ERR_SHAPE, "sizes must be in [0, 2^40]");
    if (columns > kMostColumns) return fail(CODED_ERR_UNSUPPORTED, "rows must have <= 2^33 columns");
    return CODED_OK;
}

coded_status check_tokens(const void* tok, int32_t token_bytes, int64_t n, int64_t vocab) {
    if (token_bytes != 4 && token_bytes != 8) return fail(CODED_ERR_ARG, "a token must have 4 or 8 bytes");
    if (n < 0 || n > (int64_t(1) << 31) - 1) return fail(CODED_ERR_SHAPE, "n must be in [0, 2^31 - 1]");
    if (vocab < 0 || vocab > (int64_t(1) << 31) - 2) return fail(CODED_ERR_SHAPE, "vocab must be in [0, 2^31 - 2]");
    if (n > 0 && !tok) return fail(CODED_ERR_ARG, "tok is NULL");
    if (n > 0 && !aligned(tok, token_bytes)) return fail(CODED_ERR_ARG, "tok is not aligned to its elements");
    return CODED_OK;
}

}  // namespace

extern "C" {

coded_status coded_dropout(coded_dtype dt, const void* X, int64_t q, int64_t r, int64_t ldx, double p, uint64_t seed,
                           uint64_t draw, int64_t first_row, const void* C, int64_t ldcc, void* out, int64_t ldo,
                           void* stream) {
    return guarded([&] {
        coded_status st = check_sizes(q, r);
        if (st == CODED_OK) st = check_dense("X", dt, X, q, r, ldx);
        if (st == CODED_OK && C) st = check_dense("C", dt, C, q, r, ldcc);
        if (st == CODED_OK) st = check_dense("out", dt, out, q, r, ldo);
        if (st != CODED_OK) return st;
        if (!(p >= 0.0 && p <= 1.0)) return fail(CODED_ERR_ARG, "p must be in [0, 1]");
        if (draw >> 56) return fail(CODED_ERR_ARG, "draw must be below 2^56");
        if (first_row < 0 || first_row > kMostSize) return fail(CODED_ERR_ARG, "first_row must be in [0, 2^40]");
        if (q > 0 && r > 0 && q > 1 && ((out == X && ldo != ldx) || (out == C && ldo != ldcc)))
            return fail(CODED_ERR_SHAPE, "out must have the row stride of the operand that it is");
        if (q == 0 || r == 0) return CODED_OK;
        DropoutArgs a{};
        a.X = X;
        a.C = C;
        a.out = out;
        a.q = q;
        a.r = r;
        a.ldx = ldx;
        a.ldcc = ldcc;
        a.ldo = ldo;
        a.key = coded_rng::splitmix64_output(seed, kDropoutStream << 56 | draw);
        a.least = static_cast<uint64_t>(std::nearbyint(std::ldexp(p, 32)));
        a.word0 = static_cast<uint64_t>(first_row) * (static_cast<uint64_t>(r + 1) / 2);
        a.scale = p < 1.0 ? static_cast<float>(1.0 / (1.0 - p)) : 0.0f;
        const hipError_t e = launch_dropout(a, dt == CODED_BF16, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_dropout");
    });
}

coded_status coded_embed(coded_dtype e_dt, const void* E, int64_t vocab, int64_t d, int64_t lde, const void* tok,
                         int32_t token_bytes, int64_t n, int64_t skip, double scale, coded_dtype out_dt, void* out,
                         int64_t ldo, void* stream) {
    return guarded([&] {
        coded_status st = check_tokens(tok, token_bytes, n, vocab);
        if (st == CODED_OK) st = check_sizes(0, d);
        if (st == CODED_OK) st = check_dense("E", e_dt, E, vocab, d, lde);
        if (st == CODED_OK) st = check_dense("out", out_dt, out, n, d, ldo);
        if (st != CODED_OK) return st;
        if (!(std::fabs(scale) <= kTop)) return fail(CODED_ERR_ARG, "scale must be finite in fp32");
        if (n == 0 || d == 0) return CODED_OK;
        const EmbedArgs a{E, tok, out, vocab, d, lde, n, ldo, skip, static_cast<float>(scale), token_bytes == 8, e_dt == CODED_BF16,
                          out_dt == CODED_BF16};
        const hipError_t e = launch_embed(a, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_embed");
    });
}

coded_status coded_embed_workspace(int64_t n, int64_t vocab, int64_t d, int64_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(CODED_ERR_ARG, "bytes is NULL");
        coded_status st = check_tokens(bytes, 4, n, vocab);
        if (st == CODED_OK) st = check_sizes(0, d);
        if (st != CODED_OK) return st;
        *bytes = embed_workspace_bytes(n, vocab, d);
        return CODED_OK;
    });
}

coded_status coded_embed_grad(coded_dtype g_dt, const void* G, int64_t n, int64_t d, int64_t ldg, const void* tok,
                              int32_t token_bytes, int64_t vocab, int64_t skip, double scale, double beta,
                              coded_dtype e_dt, void* dE, int64_t ldde, void* workspace, int64_t workspace_bytes,
                              void* stream) {
    return guarded([&] {
        coded_status st = check_tokens(tok, token_bytes, n, vocab);
        if (st == CODED_OK) st = check_sizes(0, d);
        if (st == CODED_OK) st = check_dense("G", g_dt, G, n, d, ldg);
        if (st == CODED_OK) st = check_dense("dE", e_dt, dE, vocab, d, ldde);
        if (st != CODED_OK) return st;
        if (!(std::fabs(scale) <= kTop && std::fabs(beta) <= kTop)) return fail(CODED_ERR_ARG, "scale and beta must be finite in fp32");
        if (vocab == 0 || d == 0) return CODED_OK;
        if (!embed_grad_fits(n, vocab, d)) return fail(CODED_ERR_UNSUPPORTED, "n * d is more than the launches reach (2^35 always fits)");
        const int64_t need = embed_workspace_bytes(n, vocab, d);
        if (need > 0) {
            if (!workspace || workspace_bytes < need)
                return fail(CODED_ERR_ARG, "the workspace must have " + std::to_string(need) + " bytes");
            if (!aligned(workspace, 16)) return fail(CODED_ERR_ARG, "the workspace must be 16-byte aligned");
        }
        const EmbedGradArgs a{G, tok, dE, vocab, d, ldg, n, ldde, skip, static_cast<float>(scale), static_cast<float>(beta),
                              token_bytes == 8, g_dt == CODED_BF16, e_dt == CODED_BF16, workspace};
        const hipError_t e = launch_embed_grad(a, static_cast<hipStream_t>(stream));
        return e == hipSuccess ? CODED_OK : hip_fail(e, "coded_embed_grad");
    });
}

}  // extern "C"
