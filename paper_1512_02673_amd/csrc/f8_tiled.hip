// Products of 8-bit matrices with many right-hand sides, in tiles on the matrix
// cores: out[i][j] = sum over blocks b of sP[b][i] sQ[b][j] (sum over b's columns
// of P[i][k] Q[j][k]).
//
// A block of 128 columns is one step.  Its codes come from memory into registers
// while the step before is computed, then into one of two halves of shared memory.
// For bf16 results a block is one 8-bit matrix instruction a tile of 16 x 16: what
// it adds up is multiplied by the scales and added to fp32 sums on the vector
// units, which run beside the matrix cores.  That instruction cuts off what lies
// more than 13 bits below the largest of eight products; a result's rounding to
// bf16 is some twenty times that.  For fp32 results the codes become bf16 values
// in registers, exactly, and meet on the bf16 instructions (half the rate), whose
// products and sums are in fp32.
//
// Q's rows lie in shared memory in an order that gives a lane 4 times TJ results
// next to each other: row j of a wave's 16 TJ is at (j % TJ) * 16 + j / TJ.
#include <algorithm>

#include "f8.h"
#include "rows.h"

namespace coded {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kThreads = 512;
constexpr int64_t kMostChain = 4096;   // blocks that one fp32 sum takes: 2^-12 of the magnitudes at the most, next to 128 terms' 2^-16 each

// How results are cut into tiles, and which tiles' sums are shared by several workgroups: the first `whole` tiles are
// one workgroup's each, the rest are split along the blocks.
struct Cut {
    int64_t bi, bj, tiles_i, tiles_j, whole, splits, per;
    __host__ __device__ int64_t rest() const { return tiles_i * tiles_j - whole; }
    __host__ __device__ int64_t groups() const { return whole + rest() * splits; }
    int64_t part_bytes() const { return splits > 1 ? rest() * splits * bi * bj * 4 : 0; }
};

struct TileArgs {
    F8Args a;
    Cut cut;
    int64_t first;   // workgroup of this launch among all
    float* part;     // [split][shared tile][place], the place as the lanes hold them
};

struct Place {
    int64_t i, j, split, shared;
};
// Workgroups go to the eight XCDs in turn: each takes a run of the whole tiles, in strips of 8 tiles of right-hand
// sides, so that what its L2 holds is used by several of them.
__device__ __forceinline__ Place place_of(const Cut& c, int64_t id) {
    const int64_t strip = id / (8 * c.tiles_j), in = id % (8 * c.tiles_j), high = lesser(8, c.tiles_i - strip * 8);
    return {strip * 8 + in % high, in / high, -1, 0};
}
__device__ __forceinline__ Place tile_place(const Cut& c, int64_t b) {
    if (b >= c.whole) {
        const int64_t rest = c.rest(), r = b - c.whole;
        Place p = place_of(c, c.whole + r % rest);
        p.split = r / rest;
        p.shared = r % rest;
        return p;
    }
    const int64_t base = c.whole / 8, more = c.whole % 8, x = b % 8;
    return place_of(c, x * base + lesser(x, more) + b / 8);
}

// A lane's results: right-hand side 16 x + li of its wave's, results (4 lk + e) TJ + y, alpha times the sums plus beta C.
template <int TI, int TJ, int WI>
__device__ __forceinline__ void put_results(const MxArgs& o, int64_t i0, int64_t j0, const f32x4_t (&acc)[TI][TJ]) {
    const int lane = threadIdx.x & 63, li = lane & 15, lk = lane >> 4, wave = threadIdx.x >> 6;
    const int64_t i1 = i0 + wave % WI * TI * 16, j1 = j0 + wave / WI * TJ * 16 + 4 * lk * TJ;
#pragma unroll
    for (int x = 0; x < TI; ++x) {
        const int64_t i = i1 + 16 * x + li;
        if (i >= o.s) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t j = j1 + e * TJ;
            if constexpr (TJ == 8) {
                float v[8];
#pragma unroll
                for (int y = 0; y < 8; ++y) v[y] = acc[x][y][e] * o.alpha;
                if (j >= o.q) continue;
                if (o.C) {
                    float c[8];
                    if (o.y_bf16)
                        row_load<true>(static_cast<const uint16_t*>(o.C) + i * o.ldcc, j, o.q, c);
                    else
                        row_load<false>(static_cast<const float*>(o.C) + i * o.ldcc, j, o.q, c);
#pragma unroll
                    for (int y = 0; y < 8; ++y) v[y] = fmaf(o.beta, c[y], v[y]);
                }
                if (o.y_bf16)
                    row_store<true>(static_cast<uint16_t*>(o.Y) + i * o.ldy, j, o.q, v);
                else
                    row_store<false>(static_cast<float*>(o.Y) + i * o.ldy, j, o.q, v);
            } else {
                if (TJ == 4 && !o.y_bf16 && j + 4 <= o.q) {
                    f32x4_t v = {acc[x][0][e], acc[x][1][e], acc[x][2 % TJ][e], acc[x][3 % TJ][e]};
                    v *= o.alpha;
                    if (o.C) {
                        const f32x4_t c = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(o.C) + i * o.ldcc + j);
#pragma unroll
                        for (int y = 0; y < 4; ++y) v[y] = fmaf(o.beta, c[y], v[y]);
                    }
                    *reinterpret_cast<f32x4_any*>(static_cast<float*>(o.Y) + i * o.ldy + j) = v;
                    continue;
                }
#pragma unroll
                for (int y = 0; y < TJ; ++y)
                    if (j + y < o.q) mx_store(o, i, j + y, acc[x][y][e]);
            }
        }
    }
}

// TI x TJ tiles of 16 x 16 a wave, WI waves along the right-hand sides and 8 / WI along the results.  ACC: by way of
// bf16.  MODE 0: Q's scales are the same for a wave's results (blocks of 128 rows), 1: P's for its right-hand sides,
// 2: neither is taken to be.
template <int TI, int TJ, int WI, bool ACC, int MODE>
__global__ __launch_bounds__(kThreads, 2) void f8_tile_kernel(TileArgs g) {
    constexpr int WJ = 8 / WI, BI = 16 * TI * WI, BJ = 16 * TJ * WJ, kRows = BI + BJ;
    constexpr int kPieces = kRows * 8 / kThreads;   // of 16 bytes a thread loads of a step
    constexpr int kPP = BI * 8 / kThreads;          // of these, P's
    static_assert(BI * 8 % kThreads == 0 && BJ * 8 % kThreads == 0 && kRows <= kThreads, "rows must split evenly over the threads");
    static_assert(MODE != 0 || 128 % (16 * TJ) == 0, "a wave's results must lie in a block");
    static_assert(MODE != 1 || 128 % (16 * TI) == 0, "a wave's right-hand sides must lie in a block");
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float* const scales = reinterpret_cast<float*>(smem + 2 * kRows * kF8Block);
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI * TI * 16, wj = wave / WI * TJ * 16;
    const MxArgs& o = g.a.o;
    const F8Mat &P = g.a.P, &Q = g.a.Q;
    const Place place = tile_place(g.cut, g.first + blockIdx.x);
    const int64_t i0 = place.i * BI, j0 = place.j * BJ;

    // What this thread loads of a step: pieces tid % 8 of rows tid / 8, 64 more, and so on.  Rows past the last one
    // read as zeros, and are not stored.
    const int row = tid >> 3, piece = tid & 7;
    const uint32_t p_from = static_cast<uint32_t>(row * P.ldc) + piece * 16, q_from = static_cast<uint32_t>(row * Q.ldc) + piece * 16;
    const auto place_in = [&](int at) { return at * kF8Block + (piece ^ ((at >> 1) & 7)) * 16; };
    const auto q_row = [](int r) { return r - r % (16 * TJ) + r % (16 * TJ) % TJ * 16 + r % (16 * TJ) / TJ; };
    const int p_to = place_in(row), q_to = place_in(BI + q_row(row));
    // 64 rows on: the same place within another wave's results, or eight rows further among 128 (another swizzle)
    [[maybe_unused]] const int q_to_odd = place_in(BI + q_row(row + 64));
    const int srow = tid < BI ? tid : lesser(tid, kRows - 1) - BI;
    const int64_t sfrom = tid < BI ? lesser(i0 + srow, o.s - 1) / P.block_rows : lesser(j0 + srow, o.q - 1) / Q.block_rows;
    const int sto = tid < BI ? srow : BI + q_row(srow);
    const int64_t t0 = place.split < 0 ? 0 : place.split * g.cut.per;
    const int64_t t1 = place.split < 0 ? g.a.blocks : lesser(t0 + g.cut.per, g.a.blocks);
    const uint8_t* p_base = P.codes + i0 * P.ldc + t0 * kF8Block;
    const uint8_t* q_base = Q.codes + j0 * Q.ldc + t0 * kF8Block;
    int64_t p_left = (o.s - 1 - i0) * P.ldc + (g.a.blocks - t0) * kF8Block, q_left = (o.q - 1 - j0) * Q.ldc + (g.a.blocks - t0) * kF8Block;
    const float* s_base = tid < BI ? P.scales + t0 * P.lds + sfrom : Q.scales + t0 * Q.lds + sfrom;
    const int64_t s_step = tid < BI ? P.lds : Q.lds;
    const uint32_t p_far = static_cast<uint32_t>(64 * P.ldc), q_far = static_cast<uint32_t>(64 * Q.ldc);
    u32x4_t next[kPieces];
    float s_next;
    const auto fetch = [&] {
        const Window p(p_base, p_left), q(q_base, q_left);
#pragma unroll
        for (int l = 0; l < kPieces; ++l) next[l] = l < kPP ? p.four(p_from + l * p_far) : q.four(q_from + (l - kPP) * q_far);
        s_next = *s_base;
        p_base += kF8Block;
        q_base += kF8Block;
        p_left -= kF8Block;
        q_left -= kF8Block;
        s_base += s_step;
    };
    const auto stage = [&](int half) {
        char* const codes = smem + half * (kRows * kF8Block);
#pragma unroll
        for (int l = 0; l < kPieces; ++l) {
            const int k = l - kPP;
            const int to = l < kPP ? p_to + l * 64 * kF8Block
                           : TJ == 8 ? (k & 1 ? q_to_odd : q_to) + k / 2 * 128 * kF8Block
                                     : q_to + k * 64 * kF8Block;
            *reinterpret_cast<u32x4_t*>(codes + to) = next[l];
        }
        if (tid < kRows) scales[half * kRows + sto] = s_next;
    };

    f32x4_t acc[TI][TJ] = {};
    // where this lane's two pieces of a row lie: rows of a tile differ in the swizzle by li alone
    const int at0 = (lk ^ ((li >> 1) & 7)) * 16 + li * kF8Block, at1 = at0 ^ 64;
    const auto compute = [&](int half) {
        const char* const codes = smem + half * (kRows * kF8Block);
        const float* const sp = scales + half * kRows + wi;
        const float* const sq = scales + half * kRows + BI + wj;
        const auto raw = [&](int row, u32x4_t (&w)[2]) {
            w[0] = *reinterpret_cast<const u32x4_t*>(codes + row * kF8Block + at0);
            w[1] = *reinterpret_cast<const u32x4_t*>(codes + row * kF8Block + at1);
        };
        float f[TI];
        [[maybe_unused]] const float one = MODE == 0 ? sq[0] : sp[0];
#pragma unroll
        for (int x = 0; x < TI; ++x) f[x] = MODE == 1 ? 1.0f : sp[16 * x + li];
        if constexpr (MODE == 0) {
#pragma unroll
            for (int x = 0; x < TI; ++x) f[x] *= one;
        }
        const auto add = [&](int x, int y, f32x4_t t, f32x4_t by) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                acc[x][y][e] = MODE == 0   ? fmaf(t[e], f[x], acc[x][y][e])
                               : MODE == 1 ? fmaf(t[e], by[e], acc[x][y][e])
                                           : fmaf(t[e] * f[x], by[e], acc[x][y][e]);
        };
        const auto scales_of = [&](int y) {
            f32x4_t by = {0.f, 0.f, 0.f, 0.f};
            if constexpr (MODE != 0) by = *reinterpret_cast<const f32x4_t*>(sq + 16 * y + 4 * lk);
            if constexpr (MODE == 1) by *= one;
            return by;
        };
        u32x4_t pw[TI][2];
#pragma unroll
        for (int x = 0; x < TI; ++x) raw(wi + 16 * x, pw[x]);
        if constexpr (ACC) {
            bf16x8 pv[TI][4];
#pragma unroll
            for (int x = 0; x < TI; ++x)
#pragma unroll
                for (int u = 0; u < 4; ++u) pv[x][u] = f8_to_bf16(pw[x][u / 2][u % 2 * 2], pw[x][u / 2][u % 2 * 2 + 1]);
#pragma unroll
            for (int y = 0; y < TJ; ++y) {
                u32x4_t qw[2];
                raw(BI + wj + 16 * y, qw);
                const f32x4_t by = scales_of(y);
                bf16x8 qv[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) qv[u] = f8_to_bf16(qw[u / 2][u % 2 * 2], qw[u / 2][u % 2 * 2 + 1]);
                f32x4_t t[TI] = {};
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int x = 0; x < TI; ++x) t[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qv[u], pv[x][u], t[x], 0, 0, 0);
#pragma unroll
                for (int x = 0; x < TI; ++x) add(x, y, t[x], by);
            }
        } else {
            // Q's operand and scales one tile row ahead, what an instruction gave two instructions behind
            u32x4_t qw[2][2];
            f32x4_t by[3], t[3];
            raw(BI + wj, qw[0]);
            by[0] = scales_of(0);
#pragma unroll
            for (int y = 0; y < TJ; ++y) {
                if (y + 1 < TJ) {
                    raw(BI + wj + 16 * (y + 1), qw[(y + 1) & 1]);
                    by[(y + 1) % 3] = scales_of(y + 1);
                }
                const i32x8_t qv = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(qw[y & 1][0], qw[y & 1][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int x = 0; x < TI; ++x) {
                    const int n = y * TI + x;
                    const i32x8_t px = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(pw[x][0], pw[x][1], 0, 1, 2, 3, 4, 5, 6, 7));
                    t[n % 3] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(qv, px, f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
                    asm volatile("" : "+v"(t[n % 3]));
                    if (n >= 2) {
                        const int px_ = (n - 2) % TI, py = (n - 2) / TI;
                        add(px_, py, t[(n - 2) % 3], by[py % 3]);
                        asm volatile("" : "+v"(acc[px_][py]));   // here, and not behind all the matrix instructions
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int n = TI * TJ - 2; n < TI * TJ; ++n) add(n % TI, n / TI, t[n % 3], by[n / TI % 3]);
        }
    };

    if (t0 < t1) {
        fetch();
        stage(0);
    }
    for (int64_t t = t0; t < t1; ++t) {
        const int half = static_cast<int>(t - t0) & 1;
        __syncthreads();
        if (t + 1 < t1) fetch();
        compute(half);
        if (t + 1 < t1) stage(half ^ 1);
    }
    if (place.split < 0) {
        put_results<TI, TJ, WI>(o, i0, j0, acc);
    } else {
        float* const part = g.part + (place.split * g.cut.rest() + place.shared) * (BI * BJ);
#pragma unroll
        for (int x = 0; x < TI; ++x)
#pragma unroll
            for (int y = 0; y < TJ; ++y) *reinterpret_cast<f32x4_t*>(part + ((x * TJ + y) * kThreads + tid) * 4) = acc[x][y];
    }
}

// The shared tiles' results from the sums of their splits, added in order.
template <int TI, int TJ, int WI>
__global__ __launch_bounds__(kThreads) void f8_shared_kernel(TileArgs g) {
    constexpr int BI = 16 * TI * WI, BJ = 16 * TJ * (8 / WI);
    const Place p = place_of(g.cut, g.cut.whole + blockIdx.x);
    f32x4_t acc[TI][TJ] = {};
    for (int64_t k = 0; k < g.cut.splits; ++k) {
        const float* const part = g.part + (k * g.cut.rest() + blockIdx.x) * (BI * BJ);
#pragma unroll
        for (int x = 0; x < TI; ++x)
#pragma unroll
            for (int y = 0; y < TJ; ++y) acc[x][y] += *reinterpret_cast<const f32x4_t*>(part + ((x * TJ + y) * kThreads + threadIdx.x) * 4);
    }
    put_results<TI, TJ, WI>(g.a.o, p.i * BI, p.j * BJ, acc);
}

constexpr int64_t lds_bytes(int64_t rows) { return 2 * rows * (kF8Block + 4); }

// Large tiles: 256 x 256 on the 8-bit instruction, 128 x 256 by way of bf16; else 64 x 128.
Cut cut_of(const F8Args& a) {
    const bool acc = !a.o.y_bf16;
    Cut best{};
    double best_us = -1;
    for (int large = 1; large >= 0; --large) {
        Cut c{};
        c.bi = large ? (acc ? 128 : 256) : 64;
        c.bj = large ? 256 : 128;
        c.tiles_i = ceil_div(a.o.s, c.bi);
        c.tiles_j = ceil_div(a.o.q, c.bj);
        const double step = large ? 2.2 : 0.5;   // us of a block
        const int64_t round = large ? 256 : 512, tiles = c.tiles_i * c.tiles_j, whole = tiles / round * round;
        for (int64_t splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (splits > a.blocks / 2 || (tiles - whole) * splits > 2 * round)) break;
            c.whole = splits > 1 ? whole : tiles;
            c.per = std::max<int64_t>(1, ceil_div(a.blocks, splits));
            c.splits = splits > 1 ? ceil_div(a.blocks, c.per) : 1;
            double us = (whole / round * a.blocks + ceil_div((tiles - whole) * c.splits, round) * c.per) * step;
            if (c.splits > 1) us += 5 + c.part_bytes() * 2 / 4e6;
            if (best_us < 0 || us < best_us) {
                best_us = us;
                best = c;
            }
        }
    }
    if (a.blocks > kMostChain) {   // every tile's sums in parts of at most kMostChain blocks
        best.whole = 0;
        best.per = std::min(best.splits > 1 ? best.per : a.blocks, kMostChain);
        best.splits = ceil_div(a.blocks, best.per);
    }
    return best;
}

template <int TI, int TJ, int WI, bool ACC, int MODE>
hipError_t launch_tiles(TileArgs g, hipStream_t st) {
    constexpr int64_t kRows = 16 * TI * WI + 16 * TJ * (8 / WI), kLds = lds_bytes(kRows);
    const auto kernel = f8_tile_kernel<TI, TJ, WI, ACC, MODE>;
    const int64_t all = g.cut.groups(), most = int64_t(1) << 22;
    for (; g.first < all; g.first += most) {
        kernel<<<dim3(static_cast<uint32_t>(lesser(most, all - g.first))), kThreads, kLds, st>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (g.cut.splits <= 1) return hipSuccess;
    if (!grid_fits(g.cut.rest(), kThreads)) return hipErrorInvalidConfiguration;
    f8_shared_kernel<TI, TJ, WI><<<dim3(static_cast<uint32_t>(g.cut.rest())), kThreads, 0, st>>>(g);
    return hipGetLastError();
}

template <int TI, int TJ, int WI, bool ACC>
hipError_t launch_large(const TileArgs& g, hipStream_t st) {
    if (g.a.Q.block_rows != 1) return launch_tiles<TI, TJ, WI, ACC, 0>(g, st);
    if (g.a.P.block_rows != 1) return launch_tiles<TI, TJ, WI, ACC, 1>(g, st);
    return launch_tiles<TI, TJ, WI, ACC, 2>(g, st);
}

}  // namespace

int64_t f8_tiled_workspace_bytes(const F8Args& a) { return cut_of(a).part_bytes(); }

hipError_t launch_f8_tiled(const F8Args& a, hipStream_t st) {
    TileArgs g{a, cut_of(a), 0, static_cast<float*>(a.o.workspace)};
    const bool acc = !a.o.y_bf16, large = g.cut.bj == 256;
    if (!large) return acc ? launch_tiles<2, 2, 2, true, 2>(g, st) : launch_tiles<2, 2, 2, false, 2>(g, st);
    return acc ? launch_large<4, 4, 2, true>(g, st) : launch_large<4, 8, 4, false>(g, st);
}

}  // namespace coded
