// Which kernel a product with a microscaled matrix takes, and the general one.
//
// The general kernel takes every size and stride: it is for matrices whose rows
// are 8 MB and more apart (A's, or a 4-bit X's that meets a 4-bit A), where the
// others' 32-bit offsets within a tile's rows do not reach (2 x 16777221, two
// columns: 0.75 s, one workgroup walking down the rows).  Each element comes by itself, so nothing is aligned or bounded.
//
// A code times its scale is a bf16 value, exactly, and so is each of the three
// pieces of an fp32 X, so the matrix cores' bf16 products are exact in fp32 and
// only the sums round.
#include "mx.h"

namespace coded {
namespace {

constexpr int kThreads = 256;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;          // right-hand sides, and results of each, a workgroup takes
constexpr int kK = 32;
constexpr int kStride = kK + 8;    // bf16 per LDS row
constexpr int kFlush = 1024 / kK;  // steps summed in one fp32 chain

// Eight consecutive values of a microscaled row into a row of a tile, zeros past `cols`.
template <int BITS>
__device__ __forceinline__ void row_piece(const MxMat& m, int64_t rows, int64_t cols, int64_t row, int64_t at,
                                          uint16_t* to, int step) {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (row < rows && at < cols) mx_eight<BITS>(m.codes + row * m.ldc, m.scales + row * m.lds, at, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i * step] = at + i < cols ? static_cast<uint16_t>(v[i / 2] >> (16 * (i & 1))) : 0;
}

// PLANES: pieces of a value of X (3: fp32).  XB: bits of a microscaled X, 0: dense.
template <int BITS, bool TRANS, int PLANES, int XB>
__global__ __launch_bounds__(kThreads) void mx_product_kernel(MxArgs a) {
    __shared__ __attribute__((aligned(16))) uint16_t Xs[PLANES][kTile * kStride];
    __shared__ __attribute__((aligned(16))) uint16_t As[kTile * kStride];
    const int64_t k = TRANS ? a.q : a.r, n = TRANS ? a.r : a.q;
    const int64_t tiles = ceil_div(a.s, kTile);
    const int64_t i0 = blockIdx.x % tiles * kTile, j0 = blockIdx.x / tiles * kTile;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, li = lane & 15, lk = lane >> 4;
    const int wi = (wave & 1) * 32, wj = (wave >> 1) * 32;
    f32x4_t sum[2][2] = {}, acc[2][2] = {};
    int steps = 0;
    for (int64_t k0 = 0; k0 < k; k0 += kK) {
        __syncthreads();
        if constexpr (XB != 0) {
            row_piece<XB>(a.XM, a.s, k, i0 + t / 4, k0 + t % 4 * 8, &Xs[0][t / 4 * kStride + t % 4 * 8], 1);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // consecutive threads on consecutive elements of X's rows
                const int ti = a.x_rows ? (t + e * kThreads) / kK : (t + e * kThreads) % kTile;
                const int tk = a.x_rows ? (t + e * kThreads) % kK : (t + e * kThreads) / kTile;
                const int64_t i = i0 + ti, kk = k0 + tk;
                const bool in = i < a.s && kk < k;
                const int64_t at = a.x_rows ? i * a.ldx + kk : kk * a.ldx + i;
                if constexpr (PLANES == 1) {
                    Xs[0][ti * kStride + tk] = in ? static_cast<const uint16_t*>(a.X)[at] : 0;
                } else {
                    uint16_t p[3];
                    split_bf16(in ? static_cast<const float*>(a.X)[at] : 0.0f, p);
#pragma unroll
                    for (int h = 0; h < 3; ++h) Xs[h][ti * kStride + tk] = p[h];
                }
            }
        }
        if constexpr (TRANS)
            row_piece<BITS>(a.A, a.q, a.r, k0 + t / 8, j0 + t % 8 * 8, &As[t % 8 * 8 * kStride + t / 8], kStride);
        else
            row_piece<BITS>(a.A, a.q, a.r, j0 + t / 4, k0 + t % 4 * 8, &As[t / 4 * kStride + t % 4 * 8], 1);
        __syncthreads();
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const bf16x8 av = *reinterpret_cast<const bf16x8*>(&As[(wj + 16 * y + li) * kStride + lk * 8]);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int h = 0; h < PLANES; ++h) {
                    const bf16x8 xv = *reinterpret_cast<const bf16x8*>(&Xs[h][(wi + 16 * x + li) * kStride + lk * 8]);
                    acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv, av, acc[x][y], 0, 0, 0);
                }
        }
        if (++steps == kFlush) {
            steps = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    sum[x][y] += acc[x][y];
                    acc[x][y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                }
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int64_t i = i0 + wi + 16 * x + 4 * lk + v, j = j0 + wj + 16 * y + li;
                if (i < a.s && j < n) mx_store(a, i, j, sum[x][y][v] + acc[x][y][v]);
            }
}

template <int BITS, bool TRANS>
hipError_t launch_bits(const MxArgs& a, hipStream_t st) {
    const int64_t blocks = ceil_div(a.s, kTile) * ceil_div(TRANS ? a.r : a.q, kTile);
    if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
    const dim3 grid(static_cast<uint32_t>(blocks));
    if (a.x_bits) {
        if constexpr (!TRANS) {
            if (a.x_bits == 4)
                mx_product_kernel<BITS, false, 1, 4><<<grid, kThreads, 0, st>>>(a);
            else
                mx_product_kernel<BITS, false, 1, 8><<<grid, kThreads, 0, st>>>(a);
        }
    } else if (a.x_bf16) {
        mx_product_kernel<BITS, TRANS, 1, 0><<<grid, kThreads, 0, st>>>(a);
    } else {
        mx_product_kernel<BITS, TRANS, 3, 0><<<grid, kThreads, 0, st>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

int64_t mx_workspace_bytes(const MxArgs& a) {
    if (mx_few_serves(a)) return mx_few_workspace_bytes(a);
    if (mx_scaled_serves(a)) return mx_scaled_workspace_bytes(a);
    return mx_tiled_serves(a) ? mx_tiled_workspace_bytes(a) : 0;
}

hipError_t launch_mx_product(const MxArgs& a, hipStream_t st) {
    if (mx_few_serves(a)) return launch_mx_few(a, st);
    if (mx_scaled_serves(a)) return launch_mx_scaled(a, st);
    if (mx_tiled_serves(a)) return launch_mx_tiled(a, st);
    if (a.A.bits == 4) return a.trans ? launch_bits<4, true>(a, st) : launch_bits<4, false>(a, st);
    return a.trans ? launch_bits<8, true>(a, st) : launch_bits<8, false>(a, st);
}

}  // namespace coded
