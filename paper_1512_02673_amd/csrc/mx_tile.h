// What the tiled products share: bounded loads, the order of the tiles, and the
// results of a matrix instruction.
#pragma once

#include <algorithm>

#include "mx_window.h"

namespace coded {
namespace {

constexpr int kThreads = 256;   // of a tile's workgroup: two waves along each of its sides
// Which tile and which split of the terms a workgroup takes.  Workgroups go to the eight XCDs in turn: each
// takes a run of tiles of its own, in strips of 8 tiles of right-hand sides, so that what its L2 holds is used
// by several of them.
struct TilePlace {
    int64_t i, j, split;
};
__device__ __forceinline__ TilePlace tile_place(int64_t tiles_i, int64_t tiles_j) {
    const int64_t total = tiles_i * tiles_j, base = total / 8, rest = total % 8;
    int64_t id = blockIdx.x % total;
    const int64_t x = id % 8;
    id = x * base + lesser(x, rest) + id / 8;
    const int64_t strip = id / (8 * tiles_j), in = id % (8 * tiles_j), high = lesser(8, tiles_i - strip * 8);
    return {strip * 8 + in % high, in / high, blockIdx.x / total};
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

// How many right-hand sides and results a tile has, and how many workgroups share its sum.
struct Cut {
    bool large;          // 128 x 256, else 64 x 128
    int64_t tiles_i, tiles_j, per, splits;   // per: steps of a split
};
inline Cut cut_tiles(int64_t s, int64_t n, int64_t steps) {
    Cut c{};
    c.large = ceil_div(s, 128) * ceil_div(n, 256) >= 256;
    c.tiles_i = ceil_div(s, c.large ? 128 : 64);
    c.tiles_j = ceil_div(n, c.large ? 256 : 128);
    const int64_t want = 512 / (c.tiles_i * c.tiles_j), most = steps / 4;
    c.splits = c.large || want < 2 || most < 2 ? 1 : want < most ? want : most;
    c.per = steps > 0 ? ceil_div(steps, c.splits) : 1;
    c.splits = steps > 0 ? ceil_div(steps, c.per) : 1;
    return c;
}

// A result's tile of four: results j .. j + 3 of side i (YROWS), or result j of sides i .. i + 3.
template <bool YROWS>
__device__ __forceinline__ void store_four(const MxArgs& a, float* part, int64_t n, int64_t i, int64_t j, f32x4_t v, bool first) {
    const int64_t side = i, have = YROWS ? n - j : a.s - i;
    if (have <= 0 || (YROWS ? i >= a.s : j >= n)) return;
    if (part) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < have) part[YROWS ? side * n + j + e : (side + e) * n + j] = v[e];
        return;
    }
    const int64_t at = YROWS ? i * a.ldy + j : j * a.ldy + i, ct = YROWS ? i * a.ldcc + j : j * a.ldcc + i;
    v *= a.alpha;
    if (a.C && first) {
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
            if (!first) v += *reinterpret_cast<const f32x4_any*>(y);
            *reinterpret_cast<f32x4_any*>(y) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < have) y[e] = first ? v[e] : y[e] + v[e];
        }
    }
}

}  // namespace
}  // namespace coded
