// Matrices in 8 bits with an fp32 scale for each block of 128 columns: what the
// host glue and the kernels share.
//
// Row t holds E4M3 codes, one a byte, in whole blocks of 128 (zeros past the last
// column).  Block b's scale is scales[b*lds + t/block_rows]: the scales of a
// tile's rows lie together, which is how a product's step takes them.
#pragma once

#include "mx_window.h"

namespace coded {

constexpr int kF8Block = 128;
constexpr float kF8Top = 448.0f;
constexpr uint32_t kF8Least = 27u << 23;   // 2^-100: the smallest magnitude that a scale is made from
// Blocks that one workgroup adds up: 4096 roundings of 2^-24 are at most 2^-12 of the sum of magnitudes.
constexpr int64_t kF8Chain = 4096;

struct F8Mat {
    uint8_t* codes;
    float* scales;
    int64_t ldc, lds;
    int64_t rows;
    int32_t block_rows;   // 1 or 128
};

// The product of P (o.s right-hand sides) and Q (o.q results of each) over o.r terms; o says what becomes of it.
struct F8Args {
    F8Mat P, Q;
    MxArgs o;
    int64_t blocks;       // of 128 terms
};

hipError_t launch_f8_quantize(const void* A, bool bf16, int64_t q, int64_t r, int64_t lda, const F8Mat* m,
                              const F8Mat* t, hipStream_t st);
hipError_t launch_f8_dequantize(const F8Mat& m, int64_t r, void* out, bool bf16, int64_t ldo, hipStream_t st);
hipError_t launch_f8_product(F8Args a, hipStream_t st);
int64_t f8_workspace_bytes(const F8Args& a);

// Few right-hand sides (f8_few.hip).
bool f8_few_serves(const F8Args& a);
int64_t f8_few_workspace_bytes(const F8Args& a);
hipError_t launch_f8_few(const F8Args& a, hipStream_t st);

// Many of both (f8_tiled.hip); results of a right-hand side in a row of Y.
int64_t f8_tiled_workspace_bytes(const F8Args& a);
hipError_t launch_f8_tiled(const F8Args& a, hipStream_t st);

#ifdef __HIPCC__
// Eight codes (two words) as a bf16 operand of the matrix instructions, exact.
__device__ __forceinline__ bf16x8 f8_to_bf16(uint32_t lo, uint32_t hi) {
    return __builtin_bit_cast(bf16x8, u32x4_t{mx_pair_bf16<8, 0>(lo, 1.0f), mx_pair_bf16<8, 1>(lo, 1.0f),
                                              mx_pair_bf16<8, 0>(hi, 1.0f), mx_pair_bf16<8, 1>(hi, 1.0f)});
}
#endif

}  // namespace coded
