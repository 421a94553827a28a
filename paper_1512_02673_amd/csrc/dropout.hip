// Dropout whose mask is a function of place: word w of the mask is SplitMix64
// output number w of the draw's generator, mix(key + (w + 1) gamma), half a word
// an element.  A thread takes eight columns of a row, four words; the state of a
// word is the one before plus gamma, so a word costs two 64-bit products.
//
// Bound: memory.  Measured: 65536 x 8192 bf16 with a residual 524 us (3.2 GB, 6.1 TB/s; a
// copy reaches 5.0), 2048 x 512 fp32 3.7.  The two products a word are hidden behind it.
#include "layers.h"

namespace coded {
namespace {

constexpr int kThreads = 256, kLogThreads = 8;
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

// SplitMix64 (Steele, Lea, Flood, OOPSLA 2014): the output of a state.
__device__ __forceinline__ uint64_t mixed(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a, RowCut cut) {
    const int64_t row = blockIdx.x / cut.pieces * cut.rows(kThreads) + (threadIdx.x >> cut.log_tpr);
    const int64_t c = ((blockIdx.x % cut.pieces << cut.log_tpr) + (threadIdx.x & ((1 << cut.log_tpr) - 1))) * 8;
    if (row >= a.q || c >= a.r) return;
    constexpr int kSize = BF16 ? 2 : 4;
    float x[8], add[8] = {};
    row_load<BF16>(static_cast<const char*>(a.X) + row * a.ldx * kSize, c, a.r, x);
    if (a.C) row_load<BF16>(static_cast<const char*>(a.C) + row * a.ldcc * kSize, c, a.r, add);
    const uint64_t words = static_cast<uint64_t>(a.r + 1) / 2;
    uint64_t z = a.key + (a.word0 + static_cast<uint64_t>(row) * words + static_cast<uint64_t>(c / 2)) * kGamma;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        z += kGamma;
        const uint64_t w = mixed(z);
        // least may be 2^32: everything is dropped
        x[2 * i] = (w & 0xFFFFFFFFu) >= a.least ? x[2 * i] * a.scale : 0.0f;
        x[2 * i + 1] = (w >> 32) >= a.least ? x[2 * i + 1] * a.scale : 0.0f;
    }
    if (a.C)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += add[i];
    row_store<BF16>(static_cast<char*>(a.out) + row * a.ldo * kSize, c, a.r, x);
}

}  // namespace

hipError_t launch_dropout(DropoutArgs a, bool bf16, hipStream_t st) {
    const RowCut cut = cut_rows(a.r, kLogThreads);
    const int64_t q = a.q, size = bf16 ? 2 : 4, step = (int64_t(1) << 23) / cut.pieces * cut.rows(kThreads);
    if (step < 1) return hipErrorInvalidConfiguration;
    for (int64_t at = 0; at < q; at += step) {
        DropoutArgs p = a;
        p.q = lesser(step, q - at);
        p.X = static_cast<const char*>(a.X) + at * a.ldx * size;
        if (a.C) p.C = static_cast<const char*>(a.C) + at * a.ldcc * size;
        p.out = static_cast<char*>(a.out) + at * a.ldo * size;
        p.word0 = a.word0 + static_cast<uint64_t>(at) * (static_cast<uint64_t>(a.r + 1) / 2);
        const dim3 grid(static_cast<uint32_t>(ceil_div(p.q, cut.rows(kThreads)) * cut.pieces));
        const auto kernel = bf16 ? dropout_kernel<true> : dropout_kernel<false>;
        kernel<<<grid, kThreads, 0, st>>>(p, cut);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace coded
