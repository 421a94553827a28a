// Products of a microscaled matrix with few right-hand sides: one vector (a
// single token, a gradient step on a vector) up to 64 columns of bf16 values.
//
// Bound: reading A's codes once; a copy of that size reads at 5.4 to 6.3 TB/s in the
// same 64- and 256-byte runs.  Measured: 65536 x 8192 in 4 bits times an fp32 vector
// 50 us (5.7 TB/s), A^T of 262144 x 4096 times one 101 (5.7), times 16 bf16 columns
// 153 (3.8), 131072 x 16384 times 64 bf16 columns 320 (3.7: there the matrix cores
// are busy 43% of the cycles and shared memory, X's operands for 32 rows a wave,
// 27%, and they take turns with the codes), 11500 x 5750 times 16 14.8 a call, two launches.
//
// The work for a code is a conversion and the
// matrix instruction, so neither shared memory nor a second copy holds codes:
// a lane loads the 16 bytes that its own part of a matrix operand is made of,
// and converts them in registers.  The order in which a sum's terms meet the
// matrix core is free as long as X is laid out in it, and that decides which
// bytes a lane loads.
//
// Columns: a right-hand side in bf16, or microscaled, is one column of the
// matrix instruction, an fp32 one is three (split_bf16), plane h of side c at
// h * s + c.  Lanes of the columns that are left over repeat column 0: a
// column's sums meet no other column's.
#include <algorithm>

#include "mx_window.h"

namespace coded {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
typedef u32x4_t u32x4_bf __attribute__((aligned(2)));
typedef u32x4_t u32x4_f __attribute__((aligned(4)));

// Eight values of a right-hand side, terms k .. k + 7 (zeros from `terms` on),
// as `planes` times eight bf16.
__device__ __forceinline__ void load_side(const MxArgs& a, int64_t side, int64_t k, int64_t terms, u32x4_t (&out)[3]) {
    if (a.x_bits) {
        uint32_t v[4] = {0u, 0u, 0u, 0u};
        if (k < terms) {   // past `terms` the codes of the last block are zero
            const uint8_t* codes = a.XM.codes + side * a.XM.ldc;
            const uint8_t* scales = a.XM.scales + side * a.XM.lds;
            if (a.x_bits == 4)
                mx_eight<4>(codes, scales, k, v);
            else
                mx_eight<8>(codes, scales, k, v);
            if (k + 8 > terms)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (k + i >= terms) v[i / 2] &= i & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
        out[0] = u32x4_t{v[0], v[1], v[2], v[3]};
        return;
    }
    const int64_t step = a.x_rows ? 1 : a.ldx;
    const int64_t at = a.x_rows ? side * a.ldx + k : k * a.ldx + side;
    if (a.x_bf16) {
        const uint16_t* p = static_cast<const uint16_t*>(a.X) + at;
        if (a.x_rows && k + 8 <= terms) {
            out[0] = *reinterpret_cast<const u32x4_bf*>(p);
        } else {
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k + i < terms ? p[i * step] : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) out[0][i] = v[2 * i] | v[2 * i + 1] << 16;
        }
        return;
    }
    const float* p = static_cast<const float*>(a.X) + at;
    float f[8];
    if (a.x_rows && k + 8 <= terms) {
        const u32x4_t lo = reinterpret_cast<const u32x4_f*>(p)[0], hi = reinterpret_cast<const u32x4_f*>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = __uint_as_float(lo[i]);
            f[4 + i] = __uint_as_float(hi[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = k + i < terms ? p[i * step] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t x[3], y[3];
        split_bf16(f[2 * i], x);
        split_bf16(f[2 * i + 1], y);
#pragma unroll
        for (int h = 0; h < 3; ++h) out[h][i] = x[h] | static_cast<uint32_t>(y[h]) << 16;
    }
}

// Values 8 U .. 8 U + 7 of a 16-byte piece of codes (32 of 4 bits, 16 of 8) as an operand of the matrix instruction.
template <int BITS, int U>
__device__ __forceinline__ bf16x8 operand(u32x4_t w, float scale) {
    u32x4_t v;
    if constexpr (BITS == 4)
        v = u32x4_t{mx_pair_bf16<4, 0>(w[U], scale), mx_pair_bf16<4, 1>(w[U], scale), mx_pair_bf16<4, 2>(w[U], scale),
                    mx_pair_bf16<4, 3>(w[U], scale)};
    else
        v = u32x4_t{mx_pair_bf16<8, 0>(w[2 * U], scale), mx_pair_bf16<8, 1>(w[2 * U], scale), mx_pair_bf16<8, 0>(w[2 * U + 1], scale),
                    mx_pair_bf16<8, 1>(w[2 * U + 1], scale)};
    return __builtin_bit_cast(bf16x8, v);
}

// ---------------------------------------------------------------- along the blocks

// Y = A X.  A wave takes RT tiles of 16 rows.  Of every step of 16 pieces (16
// bytes: 32 or 16 codes) of a row lane (li, lk) takes row li, pieces 4 t + lk: a
// load covers 64 consecutive bytes of each of 16 rows.  (Four consecutive pieces
// a lane, which are the same bytes of a step, ran at 3.4 TB/s: each load then
// touches every line of the step again.)  Part (t, u) takes values 8 u .. of the
// t-th piece.  X lies in shared memory in that order, so each operand is one
// 16-byte read, contiguous over the wave.  WK of the eight waves share their
// rows and take every WK-th step; their sums are added at the end.  Each step's
// sums start from zero and are added in fp32: a chain of 512 terms, not of all
// of them.
//
// A short X is laid out in shared memory by every workgroup for itself, before
// its loop (COLS = 0).  Else mx_order_kernel has laid it out in the workspace, in
// COLS columns, and the workgroup copies what its waves' next steps need, CP
// pieces a thread, into the other half of shared memory while they compute.
//
// All loads of the loop are issued in one straight line, a step ahead: rows past
// q, pieces past a row's end and steps past the last are addressed past the end
// of a bounded buffer, which reads as zeros and moves nothing, and the scale
// bytes past the last block are cleared.  (With branches around the loads the
// compiler waits for all that are in flight at each of them.)
template <int BITS>
constexpr int kStepOf = 16 * 128 / BITS;   // terms

// Where the eight terms from 8 g lie among pieces of eight, before the columns.
template <int BITS>
__device__ __forceinline__ int64_t ordered(int64_t g) {
    constexpr int U = 16 / BITS;   // of a piece
    const int64_t piece = g / U;
    return (piece / 4 * U + g % U) * 4 + piece % 4;
}

template <int BITS>
__global__ __launch_bounds__(256) void mx_order_kernel(MxArgs a, int planes, int64_t pieces, int cols, u32x4_t* to) {
    const int64_t id = blockIdx.x * int64_t(256) + threadIdx.x;
    const int64_t g = a.x_rows ? id % pieces : id / a.s, c = a.x_rows ? id / pieces : id % a.s;
    if (g >= pieces || c >= a.s) return;
    u32x4_t v[3];
    load_side(a, c, g * 8, a.r, v);
    u32x4_t* at = to + ordered<BITS>(g) * cols + c;
    for (int h = 0; h < planes; ++h) at[h * a.s] = h == 0 ? v[0] : h == 1 ? v[1] : v[2];
}

template <int BITS, int NT, int RT, int COLS, int CP>
__global__ __launch_bounds__(kThreads, NT == 1 ? 4 : 2) void mx_few_kernel(MxArgs a, int wk_log_, int planes, const u32x4_t* image, int64_t groups,
                                                                          int rounds_a_split, float* part) {
    constexpr int kStep = kStepOf<BITS>;
    constexpr int U = 16 / BITS;                   // operands of a piece
    constexpr int kScales = BITS == 4 ? 4 : 2;     // words of scales of a step
    constexpr uint32_t kNowhere = 0xFFFFFFF0u;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // waves on the same rows: with COLS, as many as share the pieces of X that are copied at once
    const int WK = COLS ? CP * kThreads / (kStep / 8 * (COLS ? COLS : 1)) : 1 << wk_log_;
    const int wk = wave & (WK - 1), wr = wave / WK;
    const int s = static_cast<int>(a.s), cols = planes * s, pitch = COLS ? COLS : cols;   // pitch: columns that X is laid out in
    const int rows = kWaves / WK * 16 * RT;
    const int64_t group = blockIdx.x % groups, split = blockIdx.x / groups;
    const int64_t row0 = group * rows;
    const int64_t blocks = ceil_div(a.r, kMxBlock), pieces_a = blocks * BITS / 4, steps = ceil_div(a.r, kStep);

    const int64_t have = lesser(a.q - row0, rows) - 1;
    const Window codes(a.A.codes + row0 * a.A.ldc, have * a.A.ldc + pieces_a * 16);
    const Window scales(a.A.scales + row0 * a.A.lds, have * a.A.lds + ceil_div(blocks, 4) * 4);
    uint32_t code_row[RT], scale_row[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
        const uint32_t row = (wr * RT + x) * 16 + li;
        code_row[x] = row * static_cast<uint32_t>(a.A.ldc);
        scale_row[x] = row * static_cast<uint32_t>(a.A.lds);
    }
    // Codes of the next two steps are on their way: each piece's registers take the piece two steps on as soon as
    // it is used up.
    constexpr int D = 2;
    u32x4_t w[D][RT][4];
    typedef unsigned int scales_t __attribute__((ext_vector_type(kScales)));
    scales_t sc[D][RT];
    const auto fetch_piece = [&](int step, int t, auto S) {
        const int p = step * 16 + 4 * t + lk;
        const bool in = p < static_cast<int>(pieces_a);
#pragma unroll
        for (int x = 0; x < RT; ++x) w[S.value][x][t] = codes.four(in ? code_row[x] + p * 16 : kNowhere);
    };
    const auto fetch_scales = [&](int step, auto S) {
        const uint32_t b0 = step * kScales * 4;
#pragma unroll
        for (int x = 0; x < RT; ++x) {
            const uint32_t at = step * 16 < static_cast<int>(pieces_a) ? scale_row[x] + b0 : kNowhere;   // the step's first piece is in the row
            if constexpr (BITS == 4)
                sc[S.value][x] = scales.four(at);
            else
                sc[S.value][x] = scales.two(at);
        }
    };
    const auto fetch = [&](int step, auto S) {
        fetch_scales(step, S);
#pragma unroll
        for (int t = 0; t < 4; ++t) fetch_piece(step, t, S);
    };

    int col[NT];   // byte offset of this lane's column of a column tile
#pragma unroll
    for (int n = 0; n < NT; ++n) col[n] = (16 * n + li < pitch ? 16 * n + li : 0) * 16 + lk * pitch * 16;
    const int step_bytes = kStep * pitch * 2;

    f32x4_t sum[RT][NT] = {};
    // a step's sums from X at xs; `next` is the step two rounds on
    const auto compute = [&](const char* xs, int step, int next, auto S) {
        constexpr int d = S.value;
        float scale[RT][4];
        const int left = static_cast<int>(blocks) - step * kScales * 4;
        if (left < 4 * kScales) {   // the row's last step
#pragma unroll
            for (int i = 0; i < kScales; ++i)
#pragma unroll
                for (int x = 0; x < RT; ++x) sc[d][x][i] &= left >= 4 * i + 4 ? ~0u : left <= 4 * i ? 0u : (1u << (8 * (left - 4 * i))) - 1;
        }
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                // piece 4 t + lk: byte lk of word t, or (two pieces a block) byte 2 t + lk / 2
                const uint32_t byte = BITS == 4 ? sc[d][x][t] >> (8 * lk) : sc[d][x][t / 2] >> (16 * (t & 1) + 8 * (lk >> 1));
                scale[x][t] = mx_scale(byte & 0xFFu);
            }
        fetch_scales(next, S);
        f32x4_t acc[RT][NT] = {};
        // X's operands are read one part ahead
        bf16x8 xv[2][NT];
        const auto read = [&](int p) {
#pragma unroll
            for (int n = 0; n < NT; ++n) xv[p & 1][n] = *reinterpret_cast<const bf16x8*>(xs + p * 4 * pitch * 16 + col[n]);
        };
        const auto part = [&](auto P) {
            constexpr int p = P.value;
            if constexpr (p + 1 < 4 * U) read(p + 1);
#pragma unroll
            for (int x = 0; x < RT; ++x) {
                const bf16x8 av = operand<BITS, p % U>(w[d][x][p / U], scale[x][p / U]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[x][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, xv[p & 1][n], acc[x][n], 0, 0, 0);
            }
            if constexpr (p % U == U - 1) fetch_piece(next, p / U, S);
            if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);
        };
        read(0);
        [&]<int... P>(std::integer_sequence<int, P...>) { (part(std::integral_constant<int, P>{}), ...); }(std::make_integer_sequence<int, 4 * U>{});
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int n = 0; n < NT; ++n) sum[x][n] += acc[x][n];
    };

    // Rounds of one step of each of the WK waves.  Workgroups start at different ones: in step, they would all
    // read the same columns of their rows, a whole row apart (65536 x 8192, one vector: 64 us, so 54; with every
    // workgroup at another 59.  131072 x 16384, 64 columns: 368 and 355, with every workgroup at another 327).
    const int begin = static_cast<int>(split) * rounds_a_split;
    const int rounds = static_cast<int>(lesser(rounds_a_split, ceil_div(steps, WK) - begin)), none = static_cast<int>(steps) + WK;
    const int first = NT > 1 ? blockIdx.x % rounds : ((blockIdx.x % 8) * 2 + (blockIdx.x / 8 & 1)) * rounds / 16;
    const auto round_at = [&](int i) { return begin + (first + i < rounds ? first + i : first + i - rounds); };   // i <= rounds
    const auto step_at = [&](int i) { return i < rounds ? round_at(i) * WK + wk : none; };
    typedef std::integral_constant<int, 0> even;
    typedef std::integral_constant<int, 1> odd;
    fetch(step_at(0), even{});
    fetch(step_at(1), odd{});
    if constexpr (COLS) {
        const int round = WK * step_bytes;
        const Window x(image, steps * step_bytes);
        u32x4_t xr[CP];
        const auto copy_in = [&](int64_t r) {
#pragma unroll
            for (int i = 0; i < CP; ++i) xr[i] = x.four(static_cast<uint32_t>(r * round) + (tid + i * kThreads) * 16);
        };
        const auto copy_out = [&](char* to) {
#pragma unroll
            for (int i = 0; i < CP; ++i) *reinterpret_cast<u32x4_t*>(to + (tid + i * kThreads) * 16) = xr[i];
        };
        copy_in(round_at(0));
        copy_out(smem);
        const auto turn = [&](int i, auto S) {
            __syncthreads();
            copy_in(round_at(i + 1));
            compute(smem + S.value * round + wk * step_bytes, step_at(i), step_at(i + D), S);
            copy_out(smem + (1 - S.value) * round);
        };
        for (int i = 0; i < rounds; i += 2) {
            turn(i, even{});
            if (i + 1 < rounds) turn(i + 1, odd{});
        }
    } else {
        const int pieces = static_cast<int>(steps) * (kStep / 8);
        for (int task = tid; task < pieces * s; task += kThreads) {
            const int g = a.x_rows ? task % pieces : task / s, side = a.x_rows ? task / pieces : task % s;
            u32x4_t v[3];
            load_side(a, side, g * 8, a.r, v);
            char* to = smem + (static_cast<int>(ordered<BITS>(g)) * cols + side) * 16;
            for (int h = 0; h < planes; ++h) *reinterpret_cast<u32x4_t*>(to + h * s * 16) = h == 0 ? v[0] : h == 1 ? v[1] : v[2];
        }
        __syncthreads();
        const auto turn = [&](int i, auto S) {
            const int m = step_at(i);
            if (m < steps)
                compute(smem + m * step_bytes, m, step_at(i + D), S);
            else
                fetch(step_at(i + D), S);
        };
        for (int i = 0; i < rounds; i += 2) {
            turn(i, even{});
            if (i + 1 < rounds) turn(i + 1, odd{});
        }
    }

    // the waves' tiles through shared memory: rows x columns each, then the sums over waves and pieces
    constexpr int kPitch = 16 * NT;
    float* red = reinterpret_cast<float*>(smem);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                red[(wk * rows + (wr * RT + x) * 16 + 4 * lk + v) * kPitch + 16 * n + li] = sum[x][n][v];
    __syncthreads();
    for (int task = tid; task < rows * s; task += kThreads) {
        const int t = a.y_rows ? task % rows : task / s, c = a.y_rows ? task / rows : task % s;
        if (row0 + t >= a.q) continue;
        float v = 0.0f;
        for (int h = 0; h < planes; ++h)
            for (int k = 0; k < WK; ++k) v += red[(k * rows + t) * kPitch + h * s + c];
        if (part)
            part[(split * s + c) * a.q + row0 + t] = v;
        else
            mx_store(a, c, row0 + t, v);
    }
}

// y = A x for one vector and long rows, on the vector units: a wave reads runs of 1 KB of four rows, a shape that
// memory serves better than a matrix operand's sixteen rows of 64 bytes.  A lane's 16 bytes are values of one
// block: a conversion a pair and a multiply-add a value, in fp32 with x in fp32, x's values read from shared
// memory once for the four rows.  A row's scales come as a word a lane for kSpan runs and change lanes in registers:
// loaded by the byte, with each run, those 6% of the bytes took 15% of the time.
//
// A workgroup takes `rows_wg` rows, its waves every eighth four of them, and goes over x in parts of
// `pieces_staged` runs; a row's sums of the parts before wait in shared memory.
//
// Bound: reading A.  65536 x 8192 in 4 bits 50 to 52 us (5.6 TB/s; 6.3 between that and twice the rows, the rest is
// the start), 65536 x 16384 95.6, 65536 x 4096 in 8 bits 45.1.  With two waves a SIMD in place of four 81.
//
// SIDE: where x comes from.  A contiguous fp32 or bf16 x is on its way before the first codes are (kFp32, kBf16:
// whole words), others are loaded value by value (kAny).
constexpr int kStaged = 16384;   // most columns of x in shared memory
enum Side { kAny, kFp32, kBf16 };
template <int BITS, bool NTL, Side SIDE>
__global__ __launch_bounds__(kThreads, 4) void mx_vector_kernel(MxArgs a, int rows_wg, int pieces_staged) {
    constexpr int V = 128 / BITS, kPiece = 64 * V, kRows = 4;   // values of a lane, columns of a run, rows of a wave
    constexpr int kSpan = BITS;                                 // runs whose scales one word a lane holds
    constexpr uint32_t kNowhere = 0xFFFFFFF0u;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    f32x4_t* xs = reinterpret_cast<f32x4_t*>(smem);   // [run][four values][lane]
    float* sums = reinterpret_cast<float*>(smem + pieces_staged * kPiece * 4);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row0 = blockIdx.x * static_cast<int64_t>(rows_wg);
    const int fours = static_cast<int>(ceil_div(lesser(rows_wg, a.q - row0), kRows));
    const int groups = fours > wave ? (fours - wave + kWaves - 1) / kWaves : 0;
    const int64_t blocks = ceil_div(a.r, kMxBlock), row_bytes = blocks * 4 * BITS;
    for (int64_t c0 = 0; c0 < a.r; c0 += static_cast<int64_t>(pieces_staged) * kPiece) {
        const int pieces = static_cast<int>(lesser(pieces_staged, ceil_div(a.r - c0, kPiece)));
        const bool last = c0 + static_cast<int64_t>(pieces) * kPiece >= a.r;
        const int64_t code0 = c0 * BITS / 8, scale0 = c0 / kMxBlock;
        u32x4_t w[2][kRows];
        uint32_t sc[kRows], sc_next[kRows];
        int next_group = 0, next_piece = 0;
        const auto fetch = [&](auto S) {
            const int64_t row = next_group < groups ? row0 + (wave + kWaves * next_group) * kRows : a.q;
            const int64_t have = lesser(a.q - row, kRows) - 1;
            const Window codes(a.A.codes + row * a.A.ldc + code0, have < 0 ? 0 : have * a.A.ldc + row_bytes - code0);
            const uint32_t at = next_piece * 1024 + lane * 16;
            const bool in = code0 + at < row_bytes;
#pragma unroll
            for (int e = 0; e < kRows; ++e)
                w[S.value][e] = codes.four<NTL>(in ? at + e * static_cast<uint32_t>(a.A.ldc) : kNowhere);
            if (++next_piece == pieces) {
                next_piece = 0;
                ++next_group;
            }
        };
        // the scales of a span of runs, a word a lane
        int span_group = 0, span = 0;
        const auto fetch_scales = [&] {
            const int64_t row = span_group < groups ? row0 + (wave + kWaves * span_group) * kRows : a.q;
            const int64_t have = lesser(a.q - row, kRows) - 1, words = ceil_div(blocks, 4) * 4 - scale0;
            const Window scales(a.A.scales + row * a.A.lds + scale0, have < 0 ? 0 : have * a.A.lds + words);
            const uint32_t at = span * 256 + lane * 4;
#pragma unroll
            for (int e = 0; e < kRows; ++e) sc_next[e] = scales.word(at < words ? at + e * static_cast<uint32_t>(a.A.lds) : kNowhere);
            if (++span * kSpan >= pieces) {
                span = 0;
                ++span_group;
            }
        };
        typedef std::integral_constant<int, 0> even;
        typedef std::integral_constant<int, 1> odd;
        int piece = 0, group = 0;
        constexpr int kCopies = kStaged / 4 / kThreads, kSize = SIDE == kBf16 ? 2 : 4;
        u32x4_t xr[kCopies];
        if constexpr (SIDE != kAny) {
            const Window x(static_cast<const char*>(a.X) + c0 * kSize, (a.r - c0) * kSize);
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const uint32_t from = (tid + i * kThreads) * 4 * kSize;
                if constexpr (SIDE == kFp32) {
                    xr[i] = x.four(from);
                } else {
                    const u32x2_t two = x.two(from);
                    xr[i] = u32x4_t{two[0], two[1], 0u, 0u};
                }
            }
        }
        fetch_scales();
        fetch(even{});
        fetch(odd{});
        __syncthreads();
        if constexpr (SIDE != kAny) {
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const int c = (tid + i * kThreads) * 4, in = c % kPiece;
                u32x4_t v = xr[i];
                if constexpr (SIDE == kBf16) v = u32x4_t{v[0] << 16, v[0] & 0xFFFF0000u, v[1] << 16, v[1] & 0xFFFF0000u};
                if (c < pieces * kPiece) xs[(c / kPiece * (V / 4) + in % V / 4) * 64 + in / V] = __builtin_bit_cast(f32x4_t, v);
            }
        } else {
            for (int g = tid; g < pieces * (kPiece / 8); g += kThreads) {
                u32x4_t v[3] = {};
                load_side(a, 0, c0 + g * 8, a.r, v);
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const auto plane = [&](int h) { return __uint_as_float(i & 1 ? v[h][i / 2] & 0xFFFF0000u : v[h][i / 2] << 16); };
                    f[i] = plane(0) + (plane(1) + plane(2));   // the value again, exactly
                }
                const int in = g * 8 % kPiece;
                f32x4_t* to = xs + (g * 8 / kPiece * (V / 4) + in % V / 4) * 64 + in / V;
                to[0] = f32x4_t{f[0], f[1], f[2], f[3]};
                to[64] = f32x4_t{f[4], f[5], f[6], f[7]};
            }
        }
        __syncthreads();
        float acc[kRows] = {};
        const auto turn = [&](auto S) {
            if (piece % kSpan == 0) {
                // what lies behind the row's last scale counts as no number
                const int64_t left = blocks - scale0 - piece * (kPiece / kMxBlock) - lane * 4;
#pragma unroll
                for (int e = 0; e < kRows; ++e) sc[e] = left >= 4 ? sc_next[e] : left <= 0 ? 0u : sc_next[e] & ((1u << (8 * left)) - 1);
                fetch_scales();
            }
            float scale[kRows];
            const int block = piece % kSpan * (kPiece / kMxBlock) + lane * V / kMxBlock;   // this lane's in the span
#pragma unroll
            for (int e = 0; e < kRows; ++e)
                scale[e] = mx_scale(static_cast<uint32_t>(__builtin_amdgcn_ds_bpermute(block & ~3, static_cast<int>(sc[e]))) >> (8 * (block & 3)) & 0xFFu);
            const f32x4_t* at = xs + piece * (V / 4) * 64 + lane;
#pragma unroll
            for (int word = 0; word < 4; ++word) {
                f32x4_t x[V / 16];
#pragma unroll
                for (int i = 0; i < V / 16; ++i) x[i] = at[(word * (V / 16) + i) * 64];
#pragma unroll
                for (int e = 0; e < kRows; ++e) {
                    const auto pair = [&](auto P) {
                        const mx_f32x2 v = mx_pair_f32<BITS, P.value>(w[S.value][e][word], scale[e]);
                        acc[e] = fmaf(v.x, x[P.value / 2][P.value % 2 * 2], acc[e]);
                        acc[e] = fmaf(v.y, x[P.value / 2][P.value % 2 * 2 + 1], acc[e]);
                    };
                    pair(std::integral_constant<int, 0>{});
                    pair(std::integral_constant<int, 1>{});
                    if constexpr (BITS == 4) {
                        pair(std::integral_constant<int, 2>{});
                        pair(std::integral_constant<int, 3>{});
                    }
                }
            }
            fetch(S);
            if (++piece < pieces) return;
            // the four rows' sums: half the lanes keep two rows, a quarter one, then the sixteen lanes of a row
            const bool high = lane & 32, odd_row = lane & 16;
            const float v0 = (high ? acc[2] : acc[0]) + __shfl_xor(high ? acc[0] : acc[2], 32, 64);
            const float v1 = (high ? acc[3] : acc[1]) + __shfl_xor(high ? acc[1] : acc[3], 32, 64);
            float v = (odd_row ? v1 : v0) + __shfl_xor(odd_row ? v0 : v1, 16, 64);
#pragma unroll
            for (int m = 8; m > 0; m /= 2) v += __shfl_xor(v, m, 64);
            const int row = (wave + kWaves * group) * kRows + lane / 16;
            if (lane % 16 == 0 && row0 + row < a.q) {
                if (c0 > 0) v += sums[row];
                if (last)
                    mx_store(a, 0, row0 + row, v);
                else
                    sums[row] = v;
            }
#pragma unroll
            for (int e = 0; e < kRows; ++e) acc[e] = 0.0f;
            piece = 0;
            ++group;
        };
        for (int i = 0; i < groups * pieces; i += 2) {
            turn(even{});
            if (i + 1 < groups * pieces) turn(odd{});
        }
    }
}

// ---------------------------------------------------------------- across the blocks

// Z = A^T U.  A wave takes 16 bytes of 16 neighbouring lanes' columns and walks
// down the rows, 32 a step: lane (li, lk) loads 16 bytes of rows 8 lk .. 8 lk +
// 7, which is an 8 x CW piece of A with all the terms that the matrix operand
// of each of its CW columns needs of this lane: result tile n is column n of
// every lane's piece.  The conversion makes pairs along a row and the operand
// takes pairs down a column, so two rows' pairs are exchanged by two byte
// permutations.
//
// The eight waves of a workgroup take every eighth step, workgroups take
// `per` rows each; a wave's sums go through shared memory to the workgroup's,
// and those of several workgroups to `part` (workgroup, side, column), which
// mx_join_kernel adds up in order.
//
// Rows past q repeat the last one and meet zeros of U; columns past r repeat
// the last block and are not stored.
template <int BITS, bool NTL>
__global__ __launch_bounds__(kThreads, 2) void mx_few_t_kernel(MxArgs a, int planes, int64_t per, int rows_staged, int64_t groups,
                                                               float* part) {
    constexpr int CW = 128 / BITS;     // columns of a lane
    constexpr int kCols = 16 * CW;     // and of a workgroup
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroups go to the eight XCDs in turn.  Those on the same rows share lines of scales (128 bytes
    // are eight groups' scales of a row), so each XCD takes a run of them.
    const int64_t base = gridDim.x / 8, rest = gridDim.x % 8, xcd = blockIdx.x % 8;
    const int64_t id = xcd * base + lesser(xcd, rest) + blockIdx.x / 8;
    const int64_t group = id % groups, split = id / groups;
    const int64_t t0 = split * per, t1 = lesser(t0 + per, a.q);
    const int s = static_cast<int>(a.s), cols = planes * s;
    const int64_t j0 = group * kCols;
    u32x4_t w[8];
    uint32_t sc[8];
    // rows past q read as zeros; columns past r are other bytes of A, or zeros, and are not stored
    const int64_t blocks = ceil_div(a.r, kMxBlock), c0_ = j0 * BITS / 8, b0_ = j0 / kMxBlock;
    const uint32_t code_at = static_cast<uint32_t>(8 * lk * a.A.ldc) + li * 16, scale_at = static_cast<uint32_t>(8 * lk * a.A.lds) + li * CW / kMxBlock;
    const auto fetch = [&](int64_t t) {
        const int64_t have = lesser(a.q - t, 32) - 1;
        const Window codes(a.A.codes + t * a.A.ldc + c0_, have < 0 ? 0 : have * a.A.ldc + blocks * 4 * BITS - c0_);
        const Window scales(a.A.scales + t * a.A.lds + b0_, have < 0 ? 0 : have * a.A.lds + blocks - b0_);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[e] = codes.four<NTL>(code_at + static_cast<uint32_t>(e * a.A.ldc));
            sc[e] = scales.byte(scale_at + static_cast<uint32_t>(e * a.A.lds));
        }
    };
    f32x4_t acc[CW] = {};
    const int col = (li < cols ? li : 0) * 16 + lk * cols * 16;
    int64_t mine = t0 + wave * 32;
    fetch(lesser(mine, a.q));
    for (int64_t c0 = t0; c0 < t1; c0 += rows_staged) {
        const int64_t end = lesser(c0 + rows_staged, t1);
        __syncthreads();
        const int pieces = static_cast<int>(ceil_div(end - c0, 32)) * 4;
        for (int task = tid; task < pieces * s; task += kThreads) {
            const int g = a.x_rows ? task % pieces : task / s, c = a.x_rows ? task / pieces : task % s;
            u32x4_t v[3];
            load_side(a, c, c0 + g * 8, t1, v);
            char* to = smem + (g * cols + c) * 16;
            for (int h = 0; h < planes; ++h) *reinterpret_cast<u32x4_t*>(to + h * s * 16) = h == 0 ? v[0] : h == 1 ? v[1] : v[2];
        }
        __syncthreads();
        for (; mine < end; mine += 32 * kWaves) {
            const bf16x8 u = *reinterpret_cast<const bf16x8*>(smem + static_cast<int>(mine - c0) / 8 * cols * 16 + col);
            u32x4_t cw[8];
            float scale[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                cw[e] = w[e];
                scale[e] = mx_scale(sc[e]);
            }
            fetch(mine + 32 * kWaves < t1 ? mine + 32 * kWaves : a.q);
            // a word holds 8 (4) columns: pairs of them, then down the rows
            const auto pair = [&](auto P, int word) {
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mx_pair_bf16<BITS, P.value>(cw[e][word], scale[e]);
                u32x4_t even, odd;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    even[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x05040100u);
                    odd[e] = __builtin_amdgcn_perm(v[2 * e + 1], v[2 * e], 0x07060302u);
                }
                const int n = word * (32 / BITS) + 2 * P.value;
                acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, __builtin_bit_cast(bf16x8, even), acc[n], 0, 0, 0);
                acc[n + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, __builtin_bit_cast(bf16x8, odd), acc[n + 1], 0, 0, 0);
            };
#pragma unroll
            for (int word = 0; word < 4; ++word) {
                pair(std::integral_constant<int, 0>{}, word);
                pair(std::integral_constant<int, 1>{}, word);
                if constexpr (BITS == 4) {
                    pair(std::integral_constant<int, 2>{}, word);
                    pair(std::integral_constant<int, 3>{}, word);
                }
            }
        }
    }
    // acc[n][v]: side 4 lk + v (of `cols`), column j0 + li CW + n.  One wave after
    // another would be a chain of barriers; four columns of every lane at a time
    // keep the waves' tiles within 64 x 65 floats each.
    float* red = reinterpret_cast<float*>(smem);
    constexpr int kPass = 4;   // columns of a lane a pass
    constexpr int kPitch = 16 * kPass + 1;
#pragma unroll
    for (int n0 = 0; n0 < CW; n0 += kPass) {
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kPass; ++n)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (4 * lk + v < cols) red[(wave * cols + 4 * lk + v) * kPitch + li * kPass + n] = acc[n0 + n][v];
        __syncthreads();
        for (int task = tid; task < 16 * kPass * s; task += kThreads) {
            const int p = task % (16 * kPass), c = task / (16 * kPass);
            const int64_t at = j0 + p / kPass * CW + n0 + p % kPass;
            if (at >= a.r) continue;
            float v = 0.0f;
            for (int h = 0; h < planes; ++h)
#pragma unroll
                for (int k = 0; k < kWaves; ++k) v += red[(k * cols + h * s + c) * kPitch + p];
            if (part)
                part[(split * s + c) * a.r + at] = v;
            else
                mx_store(a, c, at, v);
        }
    }
}

// Z = A^T u for one vector, in fp32 on the vector units.  As above, but each lane
// adds its 32 (16) columns by itself: a row's codes are used up by themselves, so
// the same registers take the row 256 further down at once, and with 32 sums
// instead of 128 twice as many waves have loads under way.  The sums of the four
// parts of a wave, of the eight waves and of the workgroups are added at the end.
template <int BITS, bool NTL>
__global__ __launch_bounds__(kThreads, 4) void mx_vector_t_kernel(MxArgs a, int64_t per, int rows_staged, int64_t groups, float* part) {
    constexpr int CW = 128 / BITS, kCols = 16 * CW;   // columns of a lane, and of a workgroup
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float* us = reinterpret_cast<float*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t base = gridDim.x / 8, rest = gridDim.x % 8, xcd = blockIdx.x % 8;   // as in mx_few_t_kernel
    const int64_t id = xcd * base + lesser(xcd, rest) + blockIdx.x / 8;
    const int64_t group = id % groups, split = id / groups;
    const int64_t t0 = split * per, t1 = lesser(t0 + per, a.q), j0 = group * kCols;
    const int64_t blocks = ceil_div(a.r, kMxBlock), c0_ = j0 * BITS / 8, b0_ = j0 / kMxBlock;
    const uint32_t code_at = static_cast<uint32_t>(8 * lk * a.A.ldc) + li * 16, scale_at = static_cast<uint32_t>(8 * lk * a.A.lds) + li * CW / kMxBlock;
    u32x4_t w[8];
    uint32_t sc[8];
    const auto codes_of = [&](int64_t t) {
        const int64_t have = lesser(a.q - t, 32) - 1;
        return Window(a.A.codes + t * a.A.ldc + c0_, have < 0 ? 0 : have * a.A.ldc + blocks * 4 * BITS - c0_);
    };
    const auto scales_of = [&](int64_t t) {
        const int64_t have = lesser(a.q - t, 32) - 1;
        return Window(a.A.scales + t * a.A.lds + b0_, have < 0 ? 0 : have * a.A.lds + blocks - b0_);
    };
    const auto fetch = [&](const Window& codes, const Window& scales, int e) {
        w[e] = codes.four<NTL>(code_at + static_cast<uint32_t>(e * a.A.ldc));
        sc[e] = scales.byte(scale_at + static_cast<uint32_t>(e * a.A.lds));
    };
    float acc[CW] = {};
    int64_t mine = t0 + wave * 32;
    {
        const int64_t t = lesser(mine, a.q);
        const Window codes = codes_of(t), scales = scales_of(t);
#pragma unroll
        for (int e = 0; e < 8; ++e) fetch(codes, scales, e);
    }
    for (int64_t c0 = t0; c0 < t1; c0 += rows_staged) {
        const int64_t end = lesser(c0 + rows_staged, t1);
        const int rows = static_cast<int>(ceil_div(end - c0, 32) * 32);
        __syncthreads();
        for (int i = tid; i < rows; i += kThreads) {
            const int64_t at = a.x_rows ? c0 + i : (c0 + i) * a.ldx;
            us[i] = c0 + i >= t1 ? 0.0f
                    : a.x_bf16   ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(a.X)[at]) << 16)
                                 : static_cast<const float*>(a.X)[at];
        }
        __syncthreads();
        for (; mine < end; mine += 32 * kWaves) {
            const f32x4_t* up = reinterpret_cast<const f32x4_t*>(us + static_cast<int>(mine - c0) + 8 * lk);
            const f32x4_t u[2] = {up[0], up[1]};
            const int64_t next = mine + 32 * kWaves < t1 ? mine + 32 * kWaves : a.q;
            const Window codes = codes_of(next), scales = scales_of(next);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = mx_scale(sc[e]), f = u[e / 4][e % 4];
#pragma unroll
                for (int word = 0; word < 4; ++word) {
                    const auto pair = [&](auto P) {
                        const mx_f32x2 v = mx_pair_f32<BITS, P.value>(w[e][word], s);
                        const int n = word * (32 / BITS) + 2 * P.value;
                        acc[n] = fmaf(v.x, f, acc[n]);
                        acc[n + 1] = fmaf(v.y, f, acc[n + 1]);
                    };
                    pair(std::integral_constant<int, 0>{});
                    pair(std::integral_constant<int, 1>{});
                    if constexpr (BITS == 4) {
                        pair(std::integral_constant<int, 2>{});
                        pair(std::integral_constant<int, 3>{});
                    }
                }
                fetch(codes, scales, e);
            }
        }
    }
    // eight columns of every lane at a time: 32 sums (four parts of eight waves) of 128 columns
    constexpr int kPass = 8, kPitch = 16 * kPass + 1;
    float* red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n0 = 0; n0 < CW; n0 += kPass) {
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kPass; ++n) red[(wave * 4 + lk) * kPitch + li * kPass + n] = acc[n0 + n];
        __syncthreads();
        // four threads share a column
        const int p = tid >> 2, h = tid & 3;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) v += red[(k * 4 + h) * kPitch + p];
        v += __shfl_xor(v, 1, 64);
        v += __shfl_xor(v, 2, 64);
        const int64_t at = j0 + p / kPass * CW + n0 + p % kPass;
        if (h == 0 && at < a.r) {
            if (part)
                part[split * a.r + at] = v;
            else
                mx_store(a, 0, at, v);
        }
    }
}

// Y from the partial sums of `splits` workgroups, part[split][side][result], in order.
__global__ __launch_bounds__(256) void mx_join_kernel(MxArgs a, const float* part, int64_t splits, int64_t n) {
    // a workgroup takes 32 results of one side; eight threads share each of them
    __shared__ float red[8][33];
    const int64_t tiles = ceil_div(n, 32);
    const int64_t side = blockIdx.x / tiles, at = blockIdx.x % tiles * 32 + (threadIdx.x & 31);
    const int g = threadIdx.x >> 5;
    float v = 0.0f;
    if (at < n)
#pragma unroll 4
        for (int64_t p = g; p < splits; p += 8) v += part[(p * a.s + side) * n + at];
    red[g][threadIdx.x & 31] = v;
    __syncthreads();
    if (g == 0 && at < n) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += red[i][threadIdx.x & 31];
        mx_store(a, side, at, v);
    }
}

// Codes that do not stay in the memory-side cache from call to call are loaded as such where loads take whole lines
// (A^T of 262144 x 4096 times a vector 102 us, else 118; A of 65536 x 8192 53, else 57).  In mx_few_kernel two
// loads share a line, and the second would fetch it again (65536 x 8192 54 us, so 60).
bool streamed(const MxArgs& a) { return streams(a.q * ceil_div(a.r, kMxBlock) * (4 * a.A.bits + 1)); }

// The same for many sides, 32 of them and 32 results a workgroup: read along the results and, where a row of Y
// holds the sides, turned in shared memory, so that it is written along them.
__global__ __launch_bounds__(256) void mx_join_tile_kernel(MxArgs a, const float* part, int64_t splits, int64_t n) {
    __shared__ float tile[32][33];
    const int64_t tiles = ceil_div(n, 32), j0 = blockIdx.x % tiles * 32, i0 = blockIdx.x / tiles * 32;
    const int lo = threadIdx.x & 31, hi = threadIdx.x >> 5;
    float v[4] = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i0 + hi + 8 * e < a.s && j0 + lo < n)
#pragma unroll 4
            for (int64_t p = 0; p < splits; ++p) v[e] += part[(p * a.s + i0 + hi + 8 * e) * n + j0 + lo];
    if (a.y_rows) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i0 + hi + 8 * e < a.s && j0 + lo < n) mx_store(a, i0 + hi + 8 * e, j0 + lo, v[e]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[hi + 8 * e][lo] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i0 + lo < a.s && j0 + hi + 8 * e < n) mx_store(a, i0 + lo, j0 + hi + 8 * e, tile[lo][hi + 8 * e]);
}

// One vector: mx_vector_kernel for rows of 2 KB of codes and more, or 1 KB where they do not stay in the memory-side
// cache; few long rows are cut along the terms instead.  Measured, 4 bits, mx_few_kernel and mx_vector_kernel, us:
// 65536 x 1024 11.5 14.5, x 2048 16.1 18.0, x 4096 28.0 28.3, x 8192 57.1 51.8, x 16384 117 95.6; 262144 x 1024 36.2
// 45.8, x 2048 61.7 56.2; 4096 x 16384 19.3 15.7, x 40000 24.6 34.2, 8192 x 40000 42.8 43.3, 16384 x 40000 78.5 70.9.
// An x that is loaded value by value, by every workgroup: up to 8192 columns, or where A takes longer (16384 x 16384,
// every other value 38.2 and 47.4 us, 4-bit x 300 x 16384 17.3 and 11.0; 65536 x 8192 62.9 and 57.3).
Side side_of(const MxArgs& a) {
    if (!a.x_rows || a.x_bits || (a.x_bf16 && (reinterpret_cast<uintptr_t>(a.X) % 4 || a.r % 2))) return kAny;
    return a.x_bf16 ? kBf16 : kFp32;
}
bool few_vector(const MxArgs& a) {
    const int64_t row = a.r * a.A.bits / 8;
    if (a.s != 1 || row < (streamed(a) ? 1024 : 2048)) return false;
    const bool any = side_of(a) == kAny;
    return a.r <= kStaged ? !any || a.r <= 8192 || streamed(a) : !any && a.q >= 8192;
}

int planes_of(const MxArgs& a) { return a.x_bits || a.x_bf16 ? 1 : 3; }

// How a product along the blocks is cut up.
struct FewPlan {
    int cols;            // that X is laid out in in the workspace; 0: it is not
    int rt, wk_log;      // row tiles of a wave, log2 of the waves on the same rows
    int64_t steps, lds, image_bytes;
    int64_t groups, splits, per;   // workgroups over the rows, and over the terms with `per` rounds each
    int64_t part_bytes;
};
FewPlan few_plan(const MxArgs& a) {
    FewPlan p{};
    const int64_t cols = planes_of(a) * a.s, step = a.A.bits == 4 ? 512 : 256;
    p.steps = ceil_div(a.r, step);
    const int64_t x_bytes = p.steps * step * cols * 2;
    // Every workgroup lays out X for itself while that is at most two times eight values a thread, and 64 KB.
    const bool ordered = cols > 16 || x_bytes > (64 << 10) || a.r * a.s > 16 * kThreads;
    p.cols = !ordered ? 0 : cols <= 8 ? 8 : cols <= 16 ? 16 : cols <= 32 ? 32 : 64;
    p.rt = cols <= 16 ? 1 : 2;
    p.image_bytes = p.steps * step * p.cols * 2;
    // Waves on the same rows: until there are 2048 waves, as many as there are steps.  X's pieces of a round,
    // twice, take up to 64 KB (128 KB where the registers leave a compute unit one workgroup anyway), and
    // at least one piece is each thread's.
    const int64_t tiles = ceil_div(a.q, 16 * p.rt), room = p.rt == 1 ? 64 << 10 : 128 << 10;
    if (p.cols && step / 8 * p.cols < kThreads) p.wk_log = 1;
    while (p.wk_log < 3 && (tiles << p.wk_log) < 2048 && (int64_t(2) << p.wk_log) <= p.steps &&
           2 * (step * p.cols * 2 << (p.wk_log + 1)) <= room)
        ++p.wk_log;
    const int64_t red = kWaves * 16 * p.rt * 16 * (cols <= 16 ? 1 : p.cols / 16) * 4;
    p.lds = std::max(red, p.cols ? 2 * (step * p.cols * 2 << p.wk_log) : x_bytes);
    // A round takes 0.9, 1.7 or 3.6 us with up to one workgroup a compute unit (X's 16, 32 or 64 columns).  Where
    // few rows leave units idle they share the rounds, if that saves more than adding the parts up takes
    // (16384 x 16384, 64 columns: 128 us, with four workgroups on the same rows 60).
    const int64_t rounds = ceil_div(p.steps, int64_t(1) << p.wk_log);
    p.groups = ceil_div(a.q, (kWaves >> p.wk_log) * 16 * p.rt);
    p.splits = p.cols ? std::max<int64_t>(1, std::min(256 / p.groups, rounds / 2)) : 1;
    const double us = rounds * (p.cols <= 16 ? 0.9 : p.cols == 32 ? 1.7 : 3.6);
    if (us - us / p.splits < 8 + p.splits * a.s * a.q * 4 / 2e6) p.splits = 1;
    p.per = std::max<int64_t>(1, ceil_div(rounds, p.splits));
    p.splits = std::max<int64_t>(1, ceil_div(rounds, p.per));
    p.image_bytes = (p.image_bytes + 255) / 256 * 256;
    p.part_bytes = p.splits > 1 ? p.splits * a.s * a.q * 4 : 0;
    return p;
}

template <int BITS, int NT, int RT, int COLS, int CP>
hipError_t launch_few(const MxArgs& a, const FewPlan& p, hipStream_t st) {
    if constexpr (CP * kThreads < kStepOf<BITS> / 8 * COLS) {   // less than a step of X a round
        return hipErrorInvalidConfiguration;
    } else {
        const int planes = planes_of(a);
        const int64_t blocks = p.groups * p.splits;
        if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
        u32x4_t* image = static_cast<u32x4_t*>(a.workspace);
        float* part = p.splits > 1 ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + p.image_bytes) : nullptr;
        if constexpr (COLS) {
            const int64_t pieces = p.steps * (kStepOf<BITS> / 8), threads = ceil_div(pieces * a.s, 256);
            if (!grid_fits(threads, 256)) return hipErrorInvalidConfiguration;
            mx_order_kernel<BITS><<<dim3(static_cast<uint32_t>(threads)), 256, 0, st>>>(a, planes, pieces, COLS, image);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        mx_few_kernel<BITS, NT, RT, COLS, CP><<<dim3(static_cast<uint32_t>(blocks)), kThreads, p.lds, st>>>(a, p.wk_log, planes, image, p.groups, static_cast<int>(p.per), part);
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || !part ? e : launch_mx_join(a, part, p.splits, a.q, st);
    }
}

template <int BITS>
hipError_t launch_few_cols(const MxArgs& a, hipStream_t st) {
    const FewPlan p = few_plan(a);
    // pieces of X a thread copies a round
    const int cp = static_cast<int>((kStepOf<BITS> / 8 * p.cols << p.wk_log) / kThreads);
    switch (p.cols * 16 + cp) {
        case 0: return launch_few<BITS, 1, 1, 0, 1>(a, p, st);
        case 8 * 16 + 1: return launch_few<BITS, 1, 1, 8, 1>(a, p, st);
        case 8 * 16 + 2: return launch_few<BITS, 1, 1, 8, 2>(a, p, st);
        case 8 * 16 + 4: return launch_few<BITS, 1, 1, 8, 4>(a, p, st);
        case 16 * 16 + 1: return launch_few<BITS, 1, 1, 16, 1>(a, p, st);
        case 16 * 16 + 2: return launch_few<BITS, 1, 1, 16, 2>(a, p, st);
        case 16 * 16 + 4: return launch_few<BITS, 1, 1, 16, 4>(a, p, st);
        case 32 * 16 + 2: return launch_few<BITS, 2, 2, 32, 2>(a, p, st);
        case 32 * 16 + 4: return launch_few<BITS, 2, 2, 32, 4>(a, p, st);
        case 32 * 16 + 8: return launch_few<BITS, 2, 2, 32, 8>(a, p, st);
        case 64 * 16 + 4: return launch_few<BITS, 4, 2, 64, 4>(a, p, st);
        case 64 * 16 + 8: return launch_few<BITS, 4, 2, 64, 8>(a, p, st);
        default: return hipErrorInvalidConfiguration;
    }
}

// Workgroups that share the columns of mx_few_t_kernel: about 512 in all, each
// with at least two steps for each of its waves.
int64_t t_groups(const MxArgs& a) { return ceil_div(a.r, 16 * 128 / a.A.bits); }
int64_t t_rows(const MxArgs& a) {
    const int64_t splits = std::max<int64_t>(1, (a.s == 1 ? 1024 : 512) / t_groups(a));
    const int64_t unit = 32 * kWaves;
    return std::max<int64_t>(2, ceil_div(ceil_div(a.q, splits), unit)) * unit;
}

template <int BITS>
hipError_t launch_few_t(const MxArgs& a, hipStream_t st) {
    const int planes = planes_of(a);
    const int64_t cols = planes * a.s, groups = t_groups(a), per = t_rows(a), splits = std::max<int64_t>(1, ceil_div(a.q, per));
    const int64_t unit = 32 * kWaves;
    const int64_t staged = std::min(per, std::max<int64_t>(1, (32 << 10) / (cols * 2) / unit) * unit);
    if (!grid_fits(groups * splits, kThreads)) return hipErrorInvalidConfiguration;
    constexpr int kPitch = 16 * 4 + 1;
    const int64_t lds = std::max<int64_t>(staged * cols * 2, kWaves * cols * kPitch * 4);
    float* part = splits > 1 ? static_cast<float*>(a.workspace) : nullptr;
    if (a.s == 1) {
        const int64_t rows = std::min<int64_t>(per, 8192);
        const int64_t bytes = std::max<int64_t>(rows * 4, 32 * (16 * 8 + 1) * 4);
        const auto vector = streamed(a) ? mx_vector_t_kernel<BITS, true> : mx_vector_t_kernel<BITS, false>;
        vector<<<dim3(static_cast<uint32_t>(groups * splits)), kThreads, bytes, st>>>(a, per, static_cast<int>(rows), groups, part);
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || !part ? e : launch_mx_join(a, part, splits, a.r, st);
    }
    const auto kernel = streamed(a) ? mx_few_t_kernel<BITS, true> : mx_few_t_kernel<BITS, false>;
    kernel<<<dim3(static_cast<uint32_t>(groups * splits)), kThreads, lds, st>>>(
        a, planes, per, static_cast<int>(staged), groups, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part) return e;
    return launch_mx_join(a, part, splits, a.r, st);
}

// Two workgroups of mx_vector_kernel a compute unit.
template <int BITS, bool NTL, Side SIDE>
hipError_t launch_vector_side(const MxArgs& a, hipStream_t st) {
    constexpr int kPiece = 64 * 128 / BITS;
    const int64_t rows = std::min<int64_t>(4096, ceil_div(ceil_div(a.q, 512), 4) * 4);
    const int64_t pieces = std::min<int64_t>(kStaged / kPiece, ceil_div(a.r, kPiece));
    const int64_t blocks = ceil_div(a.q, rows), lds = pieces * kPiece * 4 + (a.r > pieces * kPiece ? rows * 4 : 0);
    if (!grid_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
    mx_vector_kernel<BITS, NTL, SIDE><<<dim3(static_cast<uint32_t>(blocks)), kThreads, lds, st>>>(a, static_cast<int>(rows), static_cast<int>(pieces));
    return hipGetLastError();
}

template <int BITS>
hipError_t launch_vector(const MxArgs& a, hipStream_t st) {
    const Side side = side_of(a);
    if (streamed(a))
        return side == kAny    ? launch_vector_side<BITS, true, kAny>(a, st)
               : side == kFp32 ? launch_vector_side<BITS, true, kFp32>(a, st)
                               : launch_vector_side<BITS, true, kBf16>(a, st);
    return side == kAny    ? launch_vector_side<BITS, false, kAny>(a, st)
           : side == kFp32 ? launch_vector_side<BITS, false, kFp32>(a, st)
                           : launch_vector_side<BITS, false, kBf16>(a, st);
}

}  // namespace

hipError_t launch_mx_join(const MxArgs& a, const float* part, int64_t splits, int64_t n, hipStream_t st) {
    // Tiles where they fill the chip: else eight threads a result read the parts side by side.
    if (a.s >= 8 && ceil_div(n, 32) * ceil_div(a.s, 32) >= 512) {
        const int64_t blocks = ceil_div(n, 32) * ceil_div(a.s, 32);
        if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
        mx_join_tile_kernel<<<dim3(static_cast<uint32_t>(blocks)), 256, 0, st>>>(a, part, splits, n);
        return hipGetLastError();
    }
    const int64_t blocks = ceil_div(n, 32) * a.s;
    if (!grid_fits(blocks, 256)) return hipErrorInvalidConfiguration;
    mx_join_kernel<<<dim3(static_cast<uint32_t>(blocks)), 256, 0, st>>>(a, part, splits, n);
    return hipGetLastError();
}

// One matrix operand's columns across the blocks, four of them along.  Measured, us, these kernels and the tiles
// (mx_tiled.hip).  Across, 262144 x 4096: 2 bf16 columns 123 and 253, 16 153 and 266 (17 in tiles 288), 5 fp32 134 and
// 772 (6: 772); 8 bits, 16 columns 247 and 289; 16384 x 4096, 16: 27.4 and 26.5.  Along, 131072 x 16384: 16 bf16 columns
// 238 and 545, 64 320 and 592 (65: 742), 21 fp32 328 and 1628; 11500 x 5750: 16 13.5 and 26.4, 32 24.4 and 26.6, 64 44.2
// and 27.7; 16384 x 4096, 64: 32.5 and 24.1.  So from 33 columns on a matrix of a few thousand rows would be better off in tiles.
bool mx_few_serves(const MxArgs& a) {
    const int64_t terms = a.trans ? a.q : a.r;
    // offsets within a workgroup's rows, and steps, are 32-bit
    const int64_t most = (int64_t(1) << 31) / 256;
    return terms > 0 && a.s <= 64 && planes_of(a) * a.s <= (a.trans ? 16 : 64) && std::max(a.A.ldc, a.A.lds) < most;
}

int64_t mx_few_workspace_bytes(const MxArgs& a) {
    if (!a.trans) {
        // whatever way x lies: the sizes alone say how much, also where mx_vector_kernel needs none
        const FewPlan p = few_plan(a);
        return p.image_bytes + p.part_bytes;
    }
    const int64_t splits = ceil_div(a.q, t_rows(a));
    return splits > 1 ? splits * a.s * a.r * 4 : 0;
}

hipError_t launch_mx_few(const MxArgs& args, hipStream_t st) {
    MxArgs a = args;
    if (a.s == 1 && !a.x_rows && a.ldx == 1) {   // one contiguous right-hand side
        a.x_rows = 1;
        a.ldx = a.trans ? a.q : a.r;
    }
    if (a.trans) return a.A.bits == 4 ? launch_few_t<4>(a, st) : launch_few_t<8>(a, st);
    if (few_vector(a)) return a.A.bits == 4 ? launch_vector<4>(a, st) : launch_vector<8>(a, st);
    return a.A.bits == 4 ? launch_few_cols<4>(a, st) : launch_few_cols<8>(a, st);
}

}  // namespace coded
