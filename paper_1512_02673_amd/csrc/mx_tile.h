// What the tiled products share: bounded loads, the order of the tiles, and the
// results of a matrix instruction.
#pragma once

#include <algorithm>

#include "mx_window.h"

namespace coded {
namespace {

constexpr int kThreads = 256;   // of a tile's workgroup: two waves along each of its sides
// Terms added up in registers before the sums move to memory, 32 or 128 an addition.  Next to the magnitudes, 512
// roundings of 2^-24 are 2^-15; a bf16 result is rounded to 2^-9, and 2048 of them, 2^-13, are a sixteenth of that.
// (8192 x 33000 times 4096 tokens, bf16 results: 2.21 ms with the short chain, 2.14 with the long one and without.)
constexpr int kChain = 16384, kChainBf16 = 65536;
inline int64_t chain_steps(const MxArgs& a, int step) { return (a.y_bf16 ? kChainBf16 : kChain) / step; }
// How many right-hand sides and results a tile has, and which tiles' sums are shared by several workgroups: the
// first `whole` tiles are one workgroup's each, the rest are split along the terms.
struct Cut {
    bool large;                        // 128 x 256, else 64 x 128
    int64_t tiles_i, tiles_j, whole;
    int64_t splits, per;               // of each of the other tiles, and steps of a split
    int64_t slots;                     // whole tiles of a launch, where they have more terms than a chain: else 0
    __host__ __device__ int64_t rest() const { return tiles_i * tiles_j - whole; }
    __host__ __device__ int64_t groups() const { return whole + rest() * splits; }
    int64_t tile_bytes() const { return (large ? 128 * 256 : 64 * 128) * 4; }
    // fp32 sums of every split of every shared tile, [split][tile][place in the tile, as Y is ordered]
    int64_t part_bytes() const { return splits > 1 ? rest() * splits * tile_bytes() : 0; }
    // those, behind the whole tiles' sums of the chains so far (likewise ordered in the tile)
    int64_t sums_bytes() const { return slots * tile_bytes() + part_bytes(); }
};
constexpr int64_t kSlotBytes = int64_t(256) << 20;   // of one launch's whole tiles: four rounds of them
// Microseconds of one step of each of `groups` workgroups at once, as measured (64 terms, bf16): one to a compute
// unit, two, and as many as there are.
inline double step_us(bool large, int64_t groups) {
    if (large) return groups <= 256 ? 1.25 : groups <= 512 ? 2.0 : 2.0 * groups / 512;
    return groups <= 256 ? 0.64 : groups <= 512 ? 0.9 : 0.4 * groups / 256;
}
// Whole rounds of 512 large tiles are not split.  What is left over (2112 tiles: five rounds for the work of
// 4.1), or a product with fewer tiles than a round, is cut by the least estimated time: small tiles or large
// ones, and into how many splits, whose sums are written and read once more.  Measured (large tiles, splits 1 to
// 16, and small ones): 512 x 4096 of 4096 terms 86 57 41 46 68, 47 41 42 52 70 us; 578 x 6075 of 71240 terms in
// three planes 4321 2249 1874 (1890 with bounded chains) 1885 1892, 3043 3186 3323 3249 2682; 1000 x 1000 of 16384 terms 307 166 92 63 62,
// 163 95 67 68 72.
// `chain`: steps of the shorter chain (the workspace is asked for without the results' type).
inline Cut cut_tiles(int64_t s, int64_t n, int64_t steps, int64_t chain) {
    Cut best{};
    double best_us = -1;
    for (int large = 1; large >= 0; --large) {
        Cut c{};
        c.large = large;
        c.tiles_i = ceil_div(s, large ? 128 : 64);
        c.tiles_j = ceil_div(n, large ? 256 : 128);
        const int64_t tiles = c.tiles_i * c.tiles_j, whole = large ? tiles / 512 * 512 : 0, rest = tiles - whole;
        for (int64_t splits = 1; splits <= 64; splits *= 2) {
            if (splits > 1 && (splits > steps / 4 || rest == 0 || rest * splits > (large ? 512 : 2048))) break;
            c.whole = splits > 1 ? whole : tiles;
            c.per = steps > 0 ? ceil_div(steps, splits) : 1;
            c.splits = splits > 1 ? ceil_div(steps, c.per) : 1;
            double us = whole / 512 * steps * step_us(true, 512) + (rest > 0 ? c.per * step_us(large, rest * c.splits) : 0);
            if (c.splits > 1) us += 5 + c.part_bytes() * 2 / 5e6;
            if (best_us < 0 || us < best_us) {
                best_us = us;
                best = c;
            }
        }
    }
    if (steps > chain) best.slots = std::min(best.whole, kSlotBytes / best.tile_bytes());
    return best;
}

// f(first workgroup, workgroups) for as many launches as there are fillings of the slots.
template <class F>
hipError_t over_groups(const Cut& c, F f) {
    int64_t first = 0;
    if (c.slots)
        for (; c.whole - first > c.slots; first += c.slots) {
            const hipError_t e = f(first, c.slots);
            if (e != hipSuccess) return e;
        }
    return f(first, c.groups() - first);
}

// Which tile a workgroup takes, and which split of its terms (-1: all of them).  Workgroups go to the eight XCDs in
// turn: of the whole tiles each takes a run of its own, in strips of 8 tiles of right-hand sides, so that what
// its L2 holds is used by several of them.
struct TilePlace {
    int64_t i, j, split, shared;   // shared: its number among the tiles that are split
};
__device__ __forceinline__ TilePlace place_of(const Cut& c, int64_t id) {
    const int64_t strip = id / (8 * c.tiles_j), in = id % (8 * c.tiles_j), high = lesser(8, c.tiles_i - strip * 8);
    return {strip * 8 + in % high, in / high, -1, 0};
}
__device__ __forceinline__ TilePlace tile_place(const Cut& c, int64_t b) {
    if (b >= c.whole) {
        const int64_t rest = c.rest(), r = b - c.whole;
        TilePlace p = place_of(c, c.whole + r % rest);
        p.split = r / rest;
        p.shared = r % rest;
        return p;
    }
    const int64_t base = c.whole / 8, more = c.whole % 8, x = b % 8;
    return place_of(c, x * base + lesser(x, more) + b / 8);
}

// Shared memory, as counted: a 16-byte read serves sixteen lanes at once out of 256 bytes, lanes 0-3, 12-15 and
// 20-27 together (then 4-11, 16-19 and 28-31, and so for the upper half); a 16-byte write serves eight
// neighbours out of 128 bytes.  Operands are read with lane (li, lk) on row li: rows 0-3 and 12-15 of one lk meet
// rows 4-11 of the next.  Where those two pieces of a row differ in one bit, pieces are exchanged by row
// groups of four in the order 0, 2, 3, 1, which keeps either set of rows within pairs of that bit.
__device__ __forceinline__ int row_group(int row) {
    const int g = (row >> 2) & 3;
    return ((g ^ (g >> 1)) & 1) << 1 | g >> 1;
}

// A result's tile of four: results j .. j + 3 of side i (YROWS), or result j of sides i .. i + 3.
template <bool YROWS>
__device__ __forceinline__ void store_four(const MxArgs& a, int64_t n, int64_t i, int64_t j, f32x4_t v) {
    const int64_t have = YROWS ? n - j : a.s - i;
    if (have <= 0 || (YROWS ? i >= a.s : j >= n)) return;
    const int64_t at = YROWS ? i * a.ldy + j : j * a.ldy + i, ct = YROWS ? i * a.ldcc + j : j * a.ldcc + i;
    v *= a.alpha;
    if (a.C) {
        float c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (a.y_bf16)
                c[e] = e < have ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.C)[ct + e]) << 16) : 0.f;
            else
                c[e] = e < have ? static_cast<const float*>(a.C)[ct + e] : 0.f;
            v[e] = fmaf(a.beta, c[e], v[e]);
        }
    }
    if (a.y_bf16) {
        uint16_t* y = static_cast<uint16_t*>(a.Y) + at;
        uint16_t b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = mx_to_bf16(v[e]);
        if (have >= 4) {
            *reinterpret_cast<u32x2_any*>(y) = u32x2_t{b[0] | static_cast<uint32_t>(b[1]) << 16, b[2] | static_cast<uint32_t>(b[3]) << 16};
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < have) y[e] = b[e];
        }
    } else {
        float* y = static_cast<float*>(a.Y) + at;
        if (have >= 4) {
            *reinterpret_cast<f32x4_any*>(y) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < have) y[e] = v[e];
        }
    }
}

// The shared tiles' results from the sums of their splits, added in order.  A workgroup takes 1024 places of a tile.
template <int BI, int BJ, bool YROWS>
__global__ __launch_bounds__(kThreads) void mx_shared_tiles_kernel(MxArgs a, Cut c, const float* sums, int64_t n) {
    constexpr int kParts = BI * BJ / (4 * kThreads);
    const int64_t tile = blockIdx.x / kParts;
    const int at = (static_cast<int>(blockIdx.x % kParts) * kThreads + threadIdx.x) * 4;
    const TilePlace p = place_of(c, c.whole + tile);
    const float* from = sums + (c.slots + tile) * (BI * BJ) + at;
    f32x4_t v = *reinterpret_cast<const f32x4_t*>(from);
    for (int64_t k = 1; k < c.splits; ++k) v += *reinterpret_cast<const f32x4_t*>(from + k * c.rest() * (BI * BJ));
    const int64_t i = p.i * BI + (YROWS ? at / BJ : at % BI), j = p.j * BJ + (YROWS ? at % BJ : at / BI);
    store_four<YROWS>(a, n, i, j, v);
}

inline hipError_t launch_shared_tiles(const MxArgs& a, const Cut& c, const float* sums, int64_t n, hipStream_t st) {
    const int64_t blocks = c.rest() * ((c.large ? 128 * 256 : 64 * 128) / (4 * kThreads));
    if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
    const auto kernel = c.large ? (a.y_rows ? mx_shared_tiles_kernel<128, 256, true> : mx_shared_tiles_kernel<128, 256, false>)
                                : (a.y_rows ? mx_shared_tiles_kernel<64, 128, true> : mx_shared_tiles_kernel<64, 128, false>);
    kernel<<<dim3(static_cast<uint32_t>(blocks)), kThreads, 0, st>>>(a, c, sums, n);
    return hipGetLastError();
}

}  // namespace
}  // namespace coded
