// Products of two matrices in 4 bits, on the matrix instruction that takes codes
// and scales as they are: out[i][j] = sum over k of X[i][k] A[j][k], 128 terms
// an instruction.
//
// Lane (li, lk) of an operand holds the 16 bytes of block lk of row li and the
// block's scale.  Products are exact and sums in fp32: 384 x 512 results of
// 8192 terms were 0 to 7e-8 off in the 2-norm.  With 8-bit codes on either side
// the same instruction adds with some 14 bits (1e-5 to 5e-5 off, at any length),
// so those products take the bf16 instructions (mx_tiled.hip) at half its rate.
//
// Bound: waiting.  16384 x 8192 times 8192 columns, bf16 results, takes 870 to 910 us
// (2.4 to 2.5 PFLOP/s; the instruction alone, in a loop on registers, 8.5): the matrix cores
// are busy 27% of the cycles, shared memory 26%, and waves wait 42% of their time, at the two
// barriers of a step and for its loads, since a step's matrix work is a fourth of the
// bf16 kernel's.  The split into tiles, and the way from memory over
// registers into shared memory, are those of the products with bf16 (mx_tile.h);
// no code is converted.  Blocks past the end of a row are zeroed, what lies
// there need not be numbers; rows past the end are zeros too and not stored.
#include "mx_tile.h"

namespace coded {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kStep = 128;   // terms: four blocks

struct ScaledArgs {
    int64_t steps;
    Cut cut;
    int64_t first;   // these three as in mx_tiled.hip
    float* sums;
    int64_t chain;
};

// The rows of codes and scales that one side of a tile takes of a step.
template <int ROWS>
struct Panel {
    static constexpr int kRow = kStep / 2, kPieces = kRow / 16;
    static constexpr int kLoads = ROWS * kPieces / kThreads;
    static_assert(ROWS * kPieces % kThreads == 0 && ROWS <= kThreads, "");
    u32x4_t next[kLoads];
    uint32_t scale;

    __device__ __forceinline__ void fetch(const MxMat& m, int64_t rows, int64_t row0, int64_t blocks, int64_t t) {
        const int tid = threadIdx.x;
        const int64_t c0 = t * kRow, b0 = t * 4;
        const Window codes(m.codes + row0 * m.ldc + c0, (rows - row0 - 1) * m.ldc + blocks * 16 - c0);
        const Window scales(m.scales + row0 * m.lds + b0, (rows - row0 - 1) * m.lds + ceil_div(blocks, 4) * 4 - b0);
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
            next[l] = codes.four(static_cast<uint32_t>((tid / kPieces + l * (kThreads / kPieces)) * m.ldc + tid % kPieces * 16));
        scale = scales.word(static_cast<uint32_t>(lesser(tid, ROWS - 1) * m.lds));
        if (b0 + 4 > blocks) {
            const int have = static_cast<int>(blocks - b0);
            scale &= (1u << (8 * have)) - 1;
            if (tid % kPieces >= have)
#pragma unroll
                for (int l = 0; l < kLoads; ++l) next[l] = u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    static __device__ __forceinline__ int place(int row, int piece) {
        return row * kRow + (piece ^ row_group(row)) * 16;
    }
    __device__ __forceinline__ void stage(char* codes, uint32_t* scales) const {
        const int tid = threadIdx.x;
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
            *reinterpret_cast<u32x4_t*>(codes + place(tid / kPieces + l * (kThreads / kPieces), tid % kPieces)) = next[l];
        if (tid < ROWS) scales[tid] = scale;
    }
    // this lane's part of the operand of 16 rows, and its scale
    static __device__ __forceinline__ i32x8_t operand(const char* codes, int row, int lk) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(codes + place(row, lk));
        return i32x8_t{static_cast<int>(v[0]), static_cast<int>(v[1]), static_cast<int>(v[2]), static_cast<int>(v[3]), 0, 0, 0, 0};
    }
    static __device__ __forceinline__ int scale_of(const uint32_t* scales, int row, int lk) {
        return reinterpret_cast<const uint8_t*>(scales)[row * 4 + lk];
    }
};

template <int TI, int TJ, bool YROWS>
__global__ __launch_bounds__(kThreads, 2) void mx_scaled_kernel(MxArgs a, ScaledArgs g) {
    constexpr int BI = 32 * TI, BJ = 32 * TJ;
    constexpr int kE2M1 = 4;   // the instruction's name of the format
    typedef Panel<BI> PX;
    typedef Panel<BJ> PA;
    __shared__ __attribute__((aligned(16))) char Xs[BI * PX::kRow];
    __shared__ __attribute__((aligned(16))) char As[BJ * PA::kRow];
    __shared__ uint32_t Xe[BI], Ae[BJ];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = (wave & 1) * TI * 16, wj = (wave >> 1) * TJ * 16;
    const int64_t blocks = ceil_div(a.r, kMxBlock);
    const TilePlace place = tile_place(g.cut, g.first + blockIdx.x);
    const int64_t i0 = place.i * BI, j0 = place.j * BJ;

    PX px;
    PA pa;
    f32x4_t acc[TI][TJ] = {};
    const auto compute = [&] {
        i32x8_t xv[TI];
        int xe[TI];
#pragma unroll
        for (int x = 0; x < TI; ++x) {
            xv[x] = PX::operand(Xs, wi + 16 * x + li, lk);
            xe[x] = PX::scale_of(Xe, wi + 16 * x + li, lk);
        }
#pragma unroll
        for (int y = 0; y < TJ; ++y) {
            if (y % 2 == 0) __builtin_amdgcn_sched_barrier(0);   // reads of two operands ahead and no more: they take registers
            const i32x8_t av = PA::operand(As, wj + 16 * y + li, lk);
            const int ae = PA::scale_of(Ae, wj + 16 * y + li, lk);
#pragma unroll
            for (int x = 0; x < TI; ++x)
                acc[x][y] = YROWS ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, xv[x], acc[x][y], kE2M1, kE2M1, 0, ae, 0, xe[x])
                                  : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(xv[x], av, acc[x][y], kE2M1, kE2M1, 0, xe[x], 0, ae);
        }
    };
    const bool whole = place.split < 0;
    float* const sums = g.sums + (whole ? blockIdx.x : g.cut.slots + place.split * g.cut.rest() + place.shared) * (BI * BJ);
    // as in mx_tile_kernel
    const auto put = [&](bool first, bool last) {
        int at = tid;
        asm volatile("" : "+v"(at));
        const int l15 = at & 15, l4 = (at >> 4 & 3) * 4;
#pragma unroll
        for (int x = 0; x < TI; ++x)
#pragma unroll
            for (int y = 0; y < TJ; ++y) {
                const int ti = wi + 16 * x + (YROWS ? l15 : l4), tj = wj + 16 * y + (YROWS ? l4 : l15);
                f32x4_t* so_far = reinterpret_cast<f32x4_t*>(sums + (YROWS ? ti * BJ + tj : tj * BI + ti));
                if (!first) acc[x][y] += *so_far;
                if (whole && last)
                    store_four<YROWS>(a, a.q, i0 + ti, j0 + tj, acc[x][y]);
                else
                    *so_far = acc[x][y];
                acc[x][y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
    };
    const auto fetch = [&](int64_t t) {
        px.fetch(a.XM, a.s, i0, blocks, t);
        pa.fetch(a.A, a.q, j0, blocks, t);
    };
    const auto stage = [&] {
        px.stage(Xs, Xe);
        pa.stage(As, Ae);
    };

    int64_t t = place.split < 0 ? 0 : place.split * g.cut.per;
    const int64_t t1 = place.split < 0 ? g.steps : lesser(t + g.cut.per, g.steps);
    if (t < t1) {
        fetch(t);
        stage();
    }
    for (bool first = true;; first = false) {
        const int64_t end = lesser(t + g.chain, t1);
        for (; t < end; ++t) {
            __syncthreads();
            if (t + 1 < t1) fetch(t + 1);
            compute();
            __syncthreads();
            if (t + 1 < t1) stage();
        }
        put(first, t >= t1);
        if (t >= t1) break;
    }
}

Cut cut_of(const MxArgs& a) { return cut_tiles(a.s, a.q, ceil_div(a.r, kStep), kChain / kStep); }

}  // namespace

// Offsets within a tile's rows are 32-bit.
bool mx_scaled_serves(const MxArgs& a) {
    const int64_t most = (int64_t(1) << 31) / 256;
    return a.x_bits == 4 && a.A.bits == 4 && std::max(std::max(a.A.ldc, a.A.lds), std::max(a.XM.ldc, a.XM.lds)) < most;
}

int64_t mx_scaled_workspace_bytes(const MxArgs& a) {
    return cut_of(a).sums_bytes();
}

hipError_t launch_mx_scaled(const MxArgs& a, hipStream_t st) {
    const Cut c = cut_of(a);
    ScaledArgs g{};
    g.steps = ceil_div(a.r, kStep);
    g.cut = c;
    g.sums = static_cast<float*>(a.workspace);
    g.chain = chain_steps(a, kStep);
    if (!grid_fits(c.groups(), kThreads)) return hipErrorInvalidConfiguration;
    const auto kernel = c.large ? (a.y_rows ? mx_scaled_kernel<4, 8, true> : mx_scaled_kernel<4, 8, false>)
                                : (a.y_rows ? mx_scaled_kernel<2, 4, true> : mx_scaled_kernel<2, 4, false>);
    const hipError_t e = over_groups(c, [&](int64_t first, int64_t groups) {
        g.first = first;
        kernel<<<dim3(static_cast<uint32_t>(groups)), kThreads, 0, st>>>(a, g);
        return hipGetLastError();
    });
    if (e != hipSuccess || c.splits <= 1) return e;
    return launch_shared_tiles(a, c, g.sums, a.q, st);
}

}  // namespace coded
