// Products of 8-bit matrices with many right-hand sides, in tiles on the matrix
// cores: out[i][j] = sum over blocks b of sP[b][i] sQ[b][j] (sum over b's columns
// of P[i][k] Q[j][k]).
//
// A block of 128 columns is one step.  Its codes and scales come from memory straight
// into one of two halves of shared memory while the step before, in the other one,
// is computed; the loads go out between the matrix instructions, which would wait
// behind them if they went out at once.
//
// For bf16 results a block is two 8-bit matrix instructions a tile of 32 x 32: what they
// add up is multiplied by the scales and added to fp32 sums on the vector units,
// beside the next instructions.  Those cut off what lies more than 13 bits below the
// largest of eight products (measured: 1.5e-5 of a result in the 2-norm, 9e-5 with
// outliers); its rounding to bf16 is twenty times that.  For fp32 results the codes
// become bf16 values in registers, exactly, and meet on the bf16 instructions (half the
// rate), whose products and sums are in fp32.
//
// Q's rows lie in shared memory in an order that gives a lane 4 TJ results of a
// right-hand side next to each other: row j of a wave's 32 TJ is at (j % TJ) * 32 + j / TJ.
//
// Bound: the matrix cores and the vector units that add what they give.  Eight waves
// share 256 x 256 results, 64 x 128 a wave, or 128 x 256 by way of bf16, where
// conversions and sums take as many issue cycles as the matrix cores work; two waves a
// SIMD cover each other.  Measured in loops on one set of data, blocks of 128 on one side: bf16 results
// of 8192 x 8192 times 16384 columns 901 us (2.44 PFLOP/s, matrix cores busy 62% of the cycles; a library
// product of 8-bit matrices with one scale each 2.60), fp32 8192^3 899 (1.22; a library
// product of bf16 matrices 1.40); blocks of 1 on both sides, twice the vector work
// of the sums: bf16 8192^3 526 (2.09), fp32 8192 x 16384 times 8192 1939 (1.13).  A tile's beginning and end
// take about 8 us.  Codes by way of registers, one barrier a step, took 1092 us for the
// first, the same with 16 x 16 instructions 1126; the waves of a SIMD taking turns between
// shared memory and matrix instructions 1189; all loads at the step's start 989.
#include <algorithm>

#include "f8.h"
#include "to_shared.h"

namespace coded {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kThreads = 512;

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

// `N` neighbouring results of a right-hand side, alpha times the sums plus beta C.
template <int N, bool BF16>
__device__ __forceinline__ void put_some(const MxArgs& o, int64_t i, int64_t j, const float (&v)[N]) {
    typedef float wide_t __attribute__((ext_vector_type(N)));
    typedef wide_t wide_f __attribute__((aligned(4)));
    typedef uint16_t half_t __attribute__((ext_vector_type(N)));
    typedef half_t half_b __attribute__((aligned(2)));
    wide_t w;
#pragma unroll
    for (int y = 0; y < N; ++y) w[y] = v[y] * o.alpha;
    if (o.C) {
        wide_t c;
        if constexpr (BF16) {
            const half_t h = *reinterpret_cast<const half_b*>(static_cast<const uint16_t*>(o.C) + i * o.ldcc + j);
#pragma unroll
            for (int y = 0; y < N; ++y) c[y] = __uint_as_float(static_cast<uint32_t>(h[y]) << 16);
        } else {
            c = *reinterpret_cast<const wide_f*>(static_cast<const float*>(o.C) + i * o.ldcc + j);
        }
#pragma unroll
        for (int y = 0; y < N; ++y) w[y] = fmaf(o.beta, c[y], w[y]);
    }
    if constexpr (BF16) {
        half_t h;
#pragma unroll
        for (int y = 0; y < N; ++y) h[y] = mx_to_bf16(w[y]);
        *reinterpret_cast<half_b*>(static_cast<uint16_t*>(o.Y) + i * o.ldy + j) = h;
    } else {
        *reinterpret_cast<wide_f*>(static_cast<float*>(o.Y) + i * o.ldy + j) = w;
    }
}

// Results of the 32 right-hand sides from i0 on, a wave's 32 TJ from j0 on.  A lane has results (8 a + 4 h + b) TJ + y of
// right-hand side l31; they change places in `room` (4 TJ KB of this wave's), pieces of 16 bytes exchanged by the row,
// so that a store takes whole runs of rows.
template <int TJ, bool BF16>
__device__ __forceinline__ void put_rows(const MxArgs& o, int64_t i0, int64_t j0, const f32x4_t (&acc)[TJ][4], char* room) {
    constexpr int kRow = 128 * TJ, kPieces = kRow / 16;   // bytes and pieces of a row
    constexpr int N = BF16 ? 8 : 4, kLanes = 32 * TJ / N; // results of a lane at a time, and lanes on a row
    const int lane = threadIdx.x & 63, l31 = lane & 31, h = lane >> 5;
    const bool whole = j0 + 32 * TJ <= o.q;   // the same for the wave
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int k = 0; k < TJ; ++k) {
            f32x4_t v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[(4 * k + e) % TJ][a][(4 * k + e) / TJ];
            const int piece = (2 * a + h) * TJ + k;
            *reinterpret_cast<f32x4_t*>(room + l31 * kRow + ((piece ^ l31) & (kPieces - 1)) * 16) = v;
        }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int k = 0; k < kLanes / 2; ++k) {
        const int row = k * (64 / kLanes) + lane / kLanes, at = lane % kLanes * N;
        float v[N];
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const f32x4_t w = *reinterpret_cast<const f32x4_t*>(room + row * kRow + (((at + e) / 4 ^ row) & (kPieces - 1)) * 16);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[e + c] = w[c];
        }
        const int64_t i = i0 + row, j = j0 + at;
        if (i >= o.s) continue;
        if (whole) {
            put_some<N, BF16>(o, i, j, v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float u[1] = {v[e]};
                if (j + e < o.q) put_some<1, BF16>(o, i, j + e, u);
            }
        }
    }
}

// TI x TJ tiles of 32 x 32 a wave, WI waves along the right-hand sides and 8 / WI along the results.  ACC: by way of
// bf16.  MODE 0: Q's scales are the same for a wave's results (blocks of 128 rows), 1: P's for its right-hand sides,
// 2: neither is taken to be.
template <int TI, int TJ, int WI, bool ACC, int MODE>
__global__ __launch_bounds__(kThreads, 2) void f8_tile_kernel(TileArgs g) {
    constexpr int WJ = 8 / WI, BI = 32 * TI * WI, BJ = 32 * TJ * WJ, kRows = BI + BJ;
    constexpr int kLoads = kRows / 64;   // of 1 KB, eight rows, a wave has of a step
    constexpr int kLoading = TJ == 4 ? 5 : TJ == 2 ? 3 : 2;   // half blocks of a tile row whose products they go out between
    static_assert(kRows % 64 == 0 && kRows <= kThreads, "rows must split evenly over the waves");
    static_assert(4 * 4096 * TJ <= kRows * kF8Block, "a half of shared memory must hold four waves' results");
    static_assert(MODE != 0 || 128 % (32 * TJ) == 0, "a wave's results must lie in a block");
    static_assert(MODE != 1 || 128 % (32 * TI) == 0, "a wave's right-hand sides must lie in a block");
    // Two halves, of one step's codes and then scales each: two arrays, so that reads of one do not wait for what is
    // on its way into the other.
    __shared__ __attribute__((aligned(16))) char half0[kRows * kF8Block + kThreads * 4];
    __shared__ __attribute__((aligned(16))) char half1[kRows * kF8Block + kThreads * 4];
    const int tid = threadIdx.x, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave % WI * TI * 32, wj = wave / WI * TJ * 32;
    const MxArgs& o = g.a.o;
    const F8Mat &P = g.a.P, &Q = g.a.Q;
    const Place place = tile_place(g.cut, g.first + blockIdx.x);
    const int64_t i0 = place.i * BI, j0 = place.j * BJ;

    // Which row of the tile lies at place `at`: Q's in the order that the results come out in.  Rows past the last one
    // repeat it, and are not stored: all loads lie within the matrices.
    const auto q_row = [](int at) { return at - at % (32 * TJ) + at % 32 * TJ + at % (32 * TJ) / 32; };
    uint32_t from[kLoads];
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
        const int at = (wave * kLoads + l) * 8 + (lane >> 3), piece = (lane & 7) ^ ((at >> 1) & 7);
        from[l] = static_cast<uint32_t>(at < BI ? lesser(at, o.s - 1 - i0) * P.ldc : lesser(q_row(at - BI), o.q - 1 - j0) * Q.ldc) + piece * 16;
    }
    const int sat = wave * 64 + lane;   // the place whose scale this lane loads
    const int p_log = P.block_rows == 1 ? 0 : 7, q_log = Q.block_rows == 1 ? 0 : 7;
    const uint32_t s_from = 4 * static_cast<uint32_t>(sat < BI ? (lesser(i0 + sat, o.s - 1) >> p_log) - (i0 >> p_log)
                                                               : (lesser(j0 + q_row(lesser(sat, kRows - 1) - BI), o.q - 1) >> q_log) - (j0 >> q_log));
    const int64_t t0 = place.split < 0 ? 0 : place.split * g.cut.per;
    const int64_t t1 = place.split < 0 ? g.a.blocks : lesser(t0 + g.cut.per, g.a.blocks);
    // a wave's loads and scales are all of one side
    const uint8_t* p_base = P.codes + i0 * P.ldc + t0 * kF8Block;
    const uint8_t* q_base = Q.codes + j0 * Q.ldc + t0 * kF8Block;
    const bool s_of_p = wave * 64 < BI;
    const float* s_base = s_of_p ? P.scales + t0 * P.lds + (i0 >> p_log) : Q.scales + t0 * Q.lds + (j0 >> q_log);
    const int64_t s_step = s_of_p ? P.lds : Q.lds;
    int64_t steps = t1 - t0, ahead = steps;   // of them not fetched yet
    // Load l of a step (the last one: its scales), and on to the next step.
    const auto load = [&](char* half, int l) {
        if (l < kLoads) {
            const int at = (wave * kLoads + l) * 8;
            sixteen_to_shared(Window(at < BI ? p_base : q_base, 0xFFFFFFFF), half + at * kF8Block, from[l]);
        } else {
            four_to_shared(Window(s_base, 0xFFFFFFFF), half + kRows * kF8Block + wave * 256, s_from);
        }
    };
    const auto advance = [&] {
        if (--ahead <= 0) return;   // the last step is fetched again: loads under a condition would be waited for at once
        p_base += kF8Block;
        q_base += kF8Block;
        s_base += s_step;
    };
    const auto fetch = [&](char* half) {
#pragma unroll
        for (int l = 0; l <= kLoads; ++l) load(half, l);
        advance();
    };

    f32x4_t acc[TI][TJ][4] = {};
    // One step.  Pieces of a row lie exchanged by the row's place, (at >> 1) & 7: the 16-byte reads of sixteen lanes
    // together, eight pairs of rows, fill all banks.  This lane's pieces of a row are 2 h and 2 h + 1 of either half.
    // The next step's loads go out between the matrix instructions: at once, they would hold up the first of those.
    const auto multiply = [&](const char* half, char* other) {
        constexpr int kEach = (kLoads + 1 + kLoading - 1) / kLoading;
        const float* const sp = reinterpret_cast<const float*>(half + kRows * kF8Block) + wi;
        const float* const sq = reinterpret_cast<const float*>(half + kRows * kF8Block) + BI + wj;
        int own = l31 * kF8Block + (((2 * h) ^ (l31 >> 1)) & 7) * 16;
        asm volatile("" : "+v"(own));   // addresses are formed anew each step: kept, they would take registers from the sums
        const auto piece = [&](int row, int c) { return *reinterpret_cast<const u32x4_t*>(half + row * kF8Block + (own ^ (c / 2 * 64 + c % 2 * 16))); };
        float f[TI];
        [[maybe_unused]] float one = 1.0f;
        f32x4_t by[4];
        const auto scales_of = [&](int y) {
            if constexpr (MODE != 0)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    by[a] = *reinterpret_cast<const f32x4_t*>(sq + 32 * y + 8 * a + 4 * h);
                    if constexpr (MODE == 1) by[a] *= one;
                }
        };
        // quarters a0 .. a1 - 1 of a tile's products, by their scales, to its sums
        const auto add = [&](int x, int y, const f32x16_t& v, int a0, int a1) {
#pragma unroll
            for (int a = a0; a < a1; ++a) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = v[4 * a + e];
                    acc[x][y][a][e] = MODE == 0   ? fmaf(w, f[x], acc[x][y][a][e])
                                      : MODE == 1 ? fmaf(w, by[a][e], acc[x][y][a][e])
                                                  : fmaf(w * f[x], by[a][e], acc[x][y][a][e]);
                }
                asm volatile("" : "+v"(acc[x][y][a]));   // here, and not behind all the matrix instructions
            }
        };
        u32x4_t qw[2][2], pw[TI][4];
        qw[0][0] = piece(BI + wj, 0);
        qw[0][1] = piece(BI + wj, 1);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int x = 0; x < TI; ++x) pw[x][c] = piece(wi + 32 * x, c);
        if constexpr (MODE != 2) one = MODE == 0 ? sq[0] : sp[0];
#pragma unroll
        for (int x = 0; x < TI; ++x) f[x] = MODE == 1 ? 1.0f : sp[32 * x + l31];
        if constexpr (MODE == 0) {
#pragma unroll
            for (int x = 0; x < TI; ++x) f[x] *= one;
        }
        const f32x16_t zero = {};
        f32x16_t t[ACC && TJ > 1 ? 2 : 1][TI];
        // ACC: operand `u` of a row, eight of its codes, as bf16.
        const auto convert = [&](const u32x4_t& w, int u) {
            u32x4_t v = __builtin_bit_cast(u32x4_t, f8_to_bf16(w[u % 2 * 2], w[u % 2 * 2 + 1]));
            asm volatile("" : "+v"(v));   // between the matrix instructions, not before them
            return __builtin_bit_cast(bf16x8, v);
        };
        [[maybe_unused]] bf16x8 pv[TI][8], qv[2];
        if constexpr (ACC) {
            qv[0] = convert(qw[0][0], 0);
#pragma unroll
            for (int x = 0; x < TI; ++x) pv[x][0] = convert(pw[x][0], 0);
        }
#pragma unroll
        for (int m = 0; m < 2 * TJ; ++m) {   // tile row m / 2, half m % 2 of the block
            const int y = m / 2, u = m % 2;
            if (m + 1 < 2 * TJ) {
                qw[(m + 1) & 1][0] = piece(BI + wj + 32 * ((m + 1) / 2), (m + 1) % 2 * 2);
                qw[(m + 1) & 1][1] = piece(BI + wj + 32 * ((m + 1) / 2), (m + 1) % 2 * 2 + 1);
            }
            if constexpr (ACC) {
                // Beside each pair of instructions: the next operands' conversion, and an eighth of the tile row before.
                f32x16_t* const now = t[TJ > 1 ? y & 1 : 0];
                f32x16_t* const last = t[TJ > 1 ? (y + 1) & 1 : 0];
#pragma unroll
                for (int k = 4 * u; k < 4 * u + 4; ++k) {
#pragma unroll
                    for (int x = 0; x < TI; ++x) {
                        now[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qv[k & 1], pv[x][k], k ? now[x] : zero, 0, 0, 0);
                        asm volatile("" : "+v"(now[x]));
                        __builtin_amdgcn_sched_barrier(0);
                        if (x == 0 && k + 1 < 4 * u + 4) qv[(k + 1) & 1] = convert(qw[u][(k + 1) % 4 / 2], k + 1);
                        if (x == 0 && k + 1 == 4 * u + 4 && m + 1 < 2 * TJ) qv[(k + 1) & 1] = convert(qw[(m + 1) & 1][0], 0);
                        if (y == 0 && k + 1 < 8) pv[x][k + 1] = convert(pw[x][(k + 1) / 2], k + 1);
                        if (y > 0 && k % 2 == 0) add(x, y - 1, last[x], k / 2, k / 2 + 1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            } else {
                const i32x8_t qo = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(qw[u][0], qw[u][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int x = 0; x < TI; ++x) {
                    const i32x8_t po = __builtin_bit_cast(i32x8_t, __builtin_shufflevector(pw[x][2 * u], pw[x][2 * u + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                    if (m > 0 && u == 0) add(x, y - 1, t[0][x], 0, 4);
                    t[0][x] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(qo, po, u ? t[0][x] : zero, 0, 0, 0, 0, 0, 0);
                    asm volatile("" : "+v"(t[0][x]));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            // of this tile row, once the one before has had its own
            if (ACC ? u == 1 : u == 0) scales_of(y);
            if (m < kLoading) {
#pragma unroll
                for (int l = m * kEach; l < (m + 1) * kEach && l <= kLoads; ++l) load(other, l);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        advance();
#pragma unroll
        for (int x = 0; x < TI; ++x) add(x, TJ - 1, t[ACC && TJ > 1 ? (TJ - 1) & 1 : 0][x], 0, 4);
    };
    // What this wave loaded into shared memory is there, and every wave is here and has read what it wanted.
    const auto meet = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    if (steps & 1) {   // an odd number: one by itself, so that the loop has one way out
        fetch(half1);
        meet();
        multiply(half1, half0);
    } else if (steps) {
        fetch(half0);
    }
    for (steps &= ~int64_t(1); steps > 0; steps -= 2) {
        meet();
        multiply(half0, half1);
        meet();
        multiply(half1, half0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // shared memory is another workgroup's after this one
    if (place.split < 0) {
        __syncthreads();   // every wave has read its operands: their place is taken
        constexpr int kRoom = 4096 * TJ;   // a wave's
        char* const room = wave < 4 ? half0 + wave * kRoom : half1 + (wave - 4) * kRoom;
#pragma unroll
        for (int x = 0; x < TI; ++x) put_rows<TJ, !ACC>(o, i0 + wi + 32 * x, j0 + wj, acc[x], room);
    } else {
        float* const part = g.part + (place.split * g.cut.rest() + place.shared) * (BI * BJ);
#pragma unroll
        for (int n = 0; n < 4 * TI * TJ; ++n) *reinterpret_cast<f32x4_t*>(part + (n * kThreads + tid) * 4) = acc[n / (4 * TJ)][n / 4 % TJ][n % 4];
    }
}

// The shared tiles' results from the sums of their splits.  A workgroup takes 32 right-hand sides of one wave's results;
// its four waves add up splits in turn, in order, and the first adds up theirs.
template <int TI, int TJ, int WI, bool BF16>
__global__ __launch_bounds__(256) void f8_shared_kernel(TileArgs g) {
    constexpr int BI = 32 * TI * WI, BJ = 32 * TJ * (8 / WI), kParts = 4 * TJ;
    __shared__ __attribute__((aligned(16))) f32x4_t sums[4][kParts][64];
    const int64_t tile = blockIdx.x / (8 * TI);
    const int wave = blockIdx.x / TI % 8, x = blockIdx.x % TI, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    f32x4_t acc[TJ][4] = {};
    for (int64_t k = w; k < g.cut.splits; k += 4) {
        const float* const part = g.part + (k * g.cut.rest() + tile) * (BI * BJ) + ((x * kParts * 8 + wave) * 64 + lane) * 4;
#pragma unroll
        for (int n = 0; n < kParts; ++n) acc[n / 4][n % 4] += *reinterpret_cast<const f32x4_t*>(part + n * kThreads * 4);
    }
#pragma unroll
    for (int n = 0; n < kParts; ++n) sums[w][n][lane] = acc[n / 4][n % 4];
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int n = 0; n < kParts; ++n)
#pragma unroll
        for (int k = 1; k < 4; ++k) acc[n / 4][n % 4] += sums[k][n][lane];
    const Place p = place_of(g.cut, g.cut.whole + tile);
    put_rows<TJ, BF16>(g.a.o, p.i * BI + wave % WI * TI * 32 + 32 * x, p.j * BJ + wave / WI * TJ * 32, acc, reinterpret_cast<char*>(sums[0]));
}

// Microseconds of one block in each of `groups` workgroups at once, as measured (4096 terms): up to one a compute unit,
// and more, large ones in rounds.  `acc`: by way of bf16.
double step_us(bool large, bool acc, int64_t groups) {
    const double one = large ? (acc ? 1.4 : 1.15) : acc ? 0.6 : 0.33, full = large ? (acc ? 1.85 : 1.7) : acc ? 0.85 : 0.53;
    if (groups <= 256) return one + (full - one) * groups / 256;
    if (large) return full * ceil_div(groups, 256);
    return (acc ? 1.33 : 0.74) * (groups <= 512 ? 1.0 : groups / 512.0);
}
// Large tiles (256 x 256 on the 8-bit instruction, 128 x 256 by way of bf16) or small ones (64 x 128), and into how many
// splits what is left over from whole rounds of large tiles, or a product of less than a round, is cut: by the least
// estimated time.  A large tile's beginning and end take 8 us, a small one's 5; splits' sums 5 us and 0.35 for each MB of
// them.  Measured (large tiles with 1 to 16 splits; small ones), us, bf16 results of 4096 terms, side by side:
// 512 x 512 45 30 22 20 23; 16 13 12 14 16, 1024 x 1024 46 32 25 25 32; 17 19 18 23 32, 2048 x 2048 47 49 51 72; 28 43 47 64,
// 4096 x 4096 64 142; 102 174, 16384 x 100 45 47 48 67; 25 29 34 46; of 16384, 1000 x 1000 164 93 57 42 44; 76 50 39 43 49;
// fp32 results, 512 x 512 54 33 22 19 20; 24 18 14 15 17, 4096 x 4096 135 176; 178 228.
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
        const double edge = large ? 8 : 5;
        const int64_t tiles = c.tiles_i * c.tiles_j, whole = large ? tiles / 256 * 256 : 0, rest = tiles - whole;
        for (int64_t splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (splits > a.blocks / 2 || rest == 0 || rest * splits > 2048)) break;
            c.whole = splits > 1 ? whole : tiles;
            c.per = std::max<int64_t>(1, ceil_div(a.blocks, splits));
            c.splits = splits > 1 ? ceil_div(a.blocks, c.per) : 1;
            const int64_t groups = rest * c.splits;
            double us = whole / 256 * (a.blocks * step_us(large, acc, 256) + edge);
            if (groups > 0) us += c.per * step_us(large, acc, groups) + edge * (large ? ceil_div(groups, 256) : std::max(1.0, groups / 512.0));
            if (c.splits > 1) us += 5 + 0.35e-6 * c.part_bytes();
            if (best_us < 0 || us < best_us) {
                best_us = us;
                best = c;
            }
        }
    }
    if (a.blocks > kF8Chain) {   // every tile's sums in parts of at most kF8Chain blocks
        best.whole = 0;
        best.per = std::min(best.splits > 1 ? best.per : a.blocks, kF8Chain);
        best.splits = ceil_div(a.blocks, best.per);
    }
    return best;
}

template <int TI, int TJ, int WI, bool ACC, int MODE>
hipError_t launch_tiles(TileArgs g, hipStream_t st) {
    const auto kernel = f8_tile_kernel<TI, TJ, WI, ACC, MODE>;
    const int64_t all = g.cut.groups(), most = int64_t(1) << 22;
    for (; g.first < all; g.first += most) {
        kernel<<<dim3(static_cast<uint32_t>(lesser(most, all - g.first))), kThreads, 0, st>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (g.cut.splits <= 1) return hipSuccess;
    const int64_t joins = g.cut.rest() * 8 * TI;
    if (!grid_fits(joins, 256)) return hipErrorInvalidConfiguration;
    f8_shared_kernel<TI, TJ, WI, !ACC><<<dim3(static_cast<uint32_t>(joins)), 256, 0, st>>>(g);
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
    if (!large) return acc ? launch_tiles<1, 1, 2, true, 2>(g, st) : launch_tiles<1, 1, 2, false, 2>(g, st);
    return acc ? launch_large<2, 2, 2, true>(g, st) : launch_large<2, 4, 4, false>(g, st);
}

}  // namespace coded
