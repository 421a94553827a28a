// Dropout and embeddings: what the host glue and the kernels share.
#pragma once

#include "rows.h"

namespace coded {

struct DropoutArgs {
    const void *X, *C;      // C may be null
    void* out;
    int64_t q, r, ldx, ldcc, ldo;
    uint64_t key;           // the draw's generator
    uint64_t least;         // kept from here on: p * 2^32
    uint64_t word0;         // number of the first row's first word
    float scale;            // 1 / (1 - p)
};
hipError_t launch_dropout(DropoutArgs a, bool bf16, hipStream_t st);

struct EmbedArgs {
    const void* E;          // vocab x d
    const void* tok;
    void* out;              // n x d
    int64_t vocab, d, lde, n, ldo, skip;
    float scale;
    bool wide, e_bf16, out_bf16;
};
hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);

struct EmbedGradArgs {
    const void* G;          // n x d
    const void* tok;
    void* dE;               // vocab x d
    int64_t vocab, d, ldg, n, ldde, skip;
    float scale, beta;
    bool wide, g_bf16, e_bf16;
    void* workspace;
};
int64_t embed_workspace_bytes(int64_t n, int64_t vocab, int64_t d);
// Whether the launches take the sizes: asked before the first of them, which writes.
bool embed_grad_fits(int64_t n, int64_t vocab, int64_t d);
hipError_t launch_embed_grad(const EmbedGradArgs& a, hipStream_t st);

}  // namespace coded
