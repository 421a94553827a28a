// Products of a microscaled matrix with many right-hand sides, on the bf16
// matrix cores: out[i][j] = sum over k of P[i][k] Q[j][k], i a right-hand
// side, j a result, Q the codes' values (exact in bf16).
//
// P is X in bf16.  X is taken as it is where a row holds whole steps of a right-hand
// side, 16-byte aligned, or where a row holds one term of all of them (by columns);
// else it goes through the workspace: unpacked from codes, which is exact, or copied,
// an fp32 X as three planes (split_bf16) whose products are summed one after the
// other.  There each step's 64 terms of all sides lie together, a side's contiguous
// and padded with zeros, so that no offset within a step grows with the terms.
// Terms past the last one are zeros on one side and finite on the other; rows past
// the end of A read as zeros.
//
// Bound: the matrix cores, and the power they take: they were busy half of the
// cycles at about 2.1 GHz (operands of zeros instead of data: 10 to 18% faster, a
// library product of bf16 matrices of the same size 35%).  Four waves share a tile
// of 64 or 128 right-hand sides and 128 or 256 results, 64 x 128 a wave in the
// large one; two such workgroups on a compute unit cover each other's barriers.  A
// step's operands come from memory into registers while the step before is
// computed, then into shared memory.  Measured, bf16 results: 16384 x 4096 times
// 4099 tokens 510 us (1.08 PFLOP/s), its transpose times 4096 tokens 498 (1.10),
// 16384 x 8192 times 8192 8-bit columns 1930 (1.14), the fp32 gradient 5750 x
// 11500 of 10000 8-bit tokens 1490 (0.89).  Three planes are three times the work, the
// codes converted for each: 16384 x 4096 times 4099 fp32 tokens 1540 us (1.07), its
// transpose times 4096 1660 (0.99), 71240 x 6075 transposed times 578 1890 (0.79; a
// tenth of its tiles' sides is empty).  A library product
// of 8192^3 bf16: 1.39 to 1.45.  Tiles of 256 x 128 took 7% longer, 128 x 128 with
// three workgroups a unit 11 to 15%, 256 x 256 with one 25 to 45%; two halves of shared
// memory with one barrier a step, wave priorities, and other orders of the reads and
// matrix instructions were within 2%.
#include <algorithm>

#include "mx_tile.h"

namespace coded {
namespace {

constexpr int kStep = 64;   // terms

struct TileArgs {
    const uint16_t* P;
    int64_t pitch, step, plane; // elements between rows of a step, between steps, and between planes
    int64_t extent, shrink;     // elements from the first step's first that it may read, and how many fewer each next step may
    int32_t planes;
    int64_t steps;              // of one plane
    Cut cut;
    int64_t first;              // workgroup of this launch among all
    float* sums;                // whole tiles' sums of the chains so far, then those of the shared tiles' splits
    int64_t chain;              // steps of a chain
};

// Two waves along each side of the tile, each of TI x TJ tiles of 16 x 16.
//
// Along the blocks (mm): shared memory holds codes, and each wave converts its
// operands.  Lane (li, lk) of a step's 64 terms takes 16 lk .. 16 lk + 15, eight
// for each of two matrix instructions.  Across them (mm_t): the conversion
// comes before shared memory, which holds rows of bf16 values; the operands,
// eight terms of a column, are read transposed.  Lane (li, lk) takes terms 8 lk
// .. 8 lk + 7 of each 32.
//
// X by columns (PT: a row of X holds one term of every right-hand side) lies in
// shared memory as it is in memory, and its operands are read transposed too.
template <int BITS, bool TRANS, bool PT, int TI, int TJ, bool YROWS>
__global__ __launch_bounds__(kThreads, 2) void mx_tile_kernel(MxArgs a, TileArgs g) {
    constexpr int BI = 32 * TI, BJ = 32 * TJ;
    constexpr int kPRow = PT ? BI * 2 : kStep * 2, kPChunks = kPRow / 16;   // bytes and 16-byte pieces of a row of P's tile
    constexpr int kPLoads = BI * kStep * 2 / 16 / kThreads;
    constexpr int kQRow = TRANS ? BJ * 2 : kStep * BITS / 8;         // shared memory: [k][j] in bf16, or [j] codes
    constexpr int kQRows = TRANS ? kStep : BJ;
    constexpr int kQPieces = TRANS ? BJ * BITS / 8 / 16 : kQRow / 16;   // 16-byte pieces of codes in a row of the tile
    constexpr int kQLoads = kQRows * kQPieces / kThreads;
    constexpr int kSLoads = TRANS ? kQLoads : 1;
    __shared__ __attribute__((aligned(16))) char Ps[BI * kPRow];
    __shared__ __attribute__((aligned(16))) char Qs[kQRows * kQRow];
    __shared__ uint32_t Ss[TRANS ? 1 : BJ];
    static_assert(kQLoads >= 1 && kQRows * kQPieces % kThreads == 0, "codes must split evenly over the threads");

    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = (wave & 1) * TI * 16, wj = (wave >> 1) * TJ * 16;
    const int64_t n = TRANS ? a.r : a.q;
    const int64_t blocks = ceil_div(a.r, kMxBlock), code_row = blocks * 4 * BITS;

    const TilePlace place = tile_place(g.cut, g.first + blockIdx.x);
    const int64_t i0 = place.i * BI, j0 = place.j * BJ;

    // what this thread loads of a step: byte offsets in the tile's rows
    const uint32_t p_at = static_cast<uint32_t>(tid / kPChunks * g.pitch * 2 + tid % kPChunks * 16);
    const uint32_t q_at = static_cast<uint32_t>(tid / kQPieces * a.A.ldc + tid % kQPieces * 16);
    const uint32_t s_at = static_cast<uint32_t>(TRANS ? tid / kQPieces * a.A.lds + tid % kQPieces * 4 / BITS : lesser(tid, BJ - 1) * a.A.lds);
    u32x4_t p_next[kPLoads], q_next[kQLoads];
    uint32_t s_next[kSLoads];
    // The next step to load: where its operands begin, the bytes from there on, and its number in its plane.
    // They move on from step to step (multiplied out anew, the scalar unit's work was as long as the matrix cores').
    const int64_t t0 = place.split < 0 ? 0 : place.split * g.cut.per;
    int64_t step = t0 > 0 ? t0 % g.steps : 0;
    const int64_t q_step = TRANS ? kStep * a.A.ldc : kStep * BITS / 8, s_step = TRANS ? kStep * a.A.lds : kStep / kMxBlock;
    const int64_t q_skip = TRANS ? j0 * BITS / 8 : j0 * a.A.ldc, s_skip = TRANS ? j0 / kMxBlock : j0 * a.A.lds;
    const int64_t q_all = (a.q - 1) * a.A.ldc + code_row - q_skip;
    const int64_t s_all = (a.q - 1) * a.A.lds + (TRANS ? blocks : ceil_div(blocks, 4) * 4) - s_skip;
    const int64_t plane = t0 > 0 ? t0 / g.steps : 0, p_step = g.step;
    const uint16_t* p_base = g.P + plane * g.plane + (PT ? i0 : i0 * g.pitch) + step * p_step;
    // by columns the extent is a whole number of words, as loads are: see launch_mx_tiled
    const int64_t p_all = g.extent - (PT ? i0 : i0 * g.pitch);
    int64_t p_left = (p_all - step * g.shrink) * 2;
    const uint8_t *q_base = a.A.codes + q_skip + step * q_step, *s_base = a.A.scales + s_skip + step * s_step;
    int64_t q_left = q_all - step * q_step, s_left = s_all - step * s_step;
    const auto fetch = [&] {
        const Window p(p_base, p_left), q(q_base, q_left), s(s_base, s_left);
#pragma unroll
        for (int l = 0; l < kPLoads; ++l) p_next[l] = p.four(p_at + static_cast<uint32_t>(l * (kThreads / kPChunks) * 2 * g.pitch));
#pragma unroll
        for (int l = 0; l < kQLoads; ++l) q_next[l] = q.four(q_at + static_cast<uint32_t>(l * (kThreads / kQPieces) * a.A.ldc));
        if constexpr (TRANS) {
            // rows past q are zeros; columns past r are other bytes within A, and are not stored
#pragma unroll
            for (int l = 0; l < kQLoads; ++l) s_next[l] = s.byte(s_at + static_cast<uint32_t>(l * (kThreads / kQPieces) * a.A.lds));
        } else {
            s_next[0] = s.two_bytes(s_at);
            if (step * kStep + kStep > blocks * kMxBlock) {   // one block left: what lies behind a row is not a number for sure
                s_next[0] &= 0xFFu;
                if (tid % kQPieces >= kQPieces / 2)
#pragma unroll
                    for (int l = 0; l < kQLoads; ++l) q_next[l] = u32x4_t{0u, 0u, 0u, 0u};
            }
        }
        p_base += p_step;
        p_left -= g.shrink * 2;
        q_base += q_step;
        q_left -= q_step;
        s_base += s_step;
        s_left -= s_step;
        if (++step == g.steps) {   // the next plane
            p_base += g.plane - g.steps * p_step;
            p_left = p_all * 2;
            q_base -= g.steps * q_step;
            q_left = q_all;
            s_base -= g.steps * s_step;
            s_left = s_all;
            step = 0;
        }
    };
    // Runs of 32 bytes of a row that is read transposed, exchanged so that two neighbouring parts of a wave, four
    // rows each, read all banks: their rows are 8 (across the blocks) or 16 (along them) apart.  Rows of 128
    // bytes fill the banks in pairs.
    const auto run_swizzle = [](int row, int pitch) {
        const int far = TRANS ? (row >> 3) & 1 : (row >> 4) & 1;
        return pitch >= 256 ? (row & 3) | far << 2 : ((row >> 1) & 1) | far << 1;
    };
    const auto transposed = [&](const char* tile, int pitch, int run, int u) {
        typedef __attribute__((address_space(3))) s16x4_t lds4;
        const int row = (TRANS ? 32 * u + 8 * lk : 16 * lk + 8 * u) + (li >> 2);
        const char* at = tile + row * pitch + (run ^ run_swizzle(row, pitch)) * 32 + (li & 3) * 8;
        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(at));
        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(at + 4 * pitch));   // the same runs there
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // two rows of P fill the banks; a lane's pieces are 2 lk + u, or 4 u + lk
    const auto p_swizzle = [](int row) { return TRANS ? (row >> 1) & 7 : row_group(row) << 1 | ((row >> 1) & 1); };
    const auto stage = [&] {
#pragma unroll
        for (int l = 0; l < kPLoads; ++l) {
            const int id_ = tid + l * kThreads, row = id_ / kPChunks, c = id_ % kPChunks;
            const int at = !PT ? c ^ p_swizzle(row) : c ^ run_swizzle(row, kPRow) << 1;
            *reinterpret_cast<u32x4_t*>(Ps + row * kPRow + at * 16) = p_next[l];
        }
#pragma unroll
        for (int l = 0; l < kQLoads; ++l) {
            const int id_ = tid + l * kThreads, row = id_ / kQPieces, c = id_ % kQPieces;
            char* to = Qs + row * kQRow;
            if constexpr (!TRANS) {
                const int at = BITS == 4 ? c ^ ((row >> 3) & 1) : c ^ row_group(row);
                *reinterpret_cast<u32x4_t*>(to + at * 16) = q_next[l];
            } else {
                const float s = mx_scale(s_next[l]);
                const int f = run_swizzle(row, kQRow);
                // a lane's pieces of eight values in an order of its own, so that eight neighbours write 128 bytes of banks
                const int turn = BITS == 4 ? (c >> 1) & 3 : (c >> 2) & 1;
                u32x4_t w = q_next[l];
                if constexpr (BITS == 4) {
                    w = turn & 1 ? u32x4_t{w[1], w[0], w[3], w[2]} : w;
                    w = turn & 2 ? u32x4_t{w[2], w[3], w[0], w[1]} : w;
                } else {
                    w = turn ? u32x4_t{w[2], w[3], w[0], w[1]} : w;
                }
#pragma unroll
                for (int e = 0; e < 16 / BITS; ++e) {
                    u32x4_t v;
                    if constexpr (BITS == 4)
                        v = u32x4_t{mx_pair_bf16<4, 0>(w[e], s), mx_pair_bf16<4, 1>(w[e], s), mx_pair_bf16<4, 2>(w[e], s),
                                    mx_pair_bf16<4, 3>(w[e], s)};
                    else
                        v = u32x4_t{mx_pair_bf16<8, 0>(w[2 * e], s), mx_pair_bf16<8, 1>(w[2 * e], s), mx_pair_bf16<8, 0>(w[2 * e + 1], s),
                                    mx_pair_bf16<8, 1>(w[2 * e + 1], s)};
                    const int at = e ^ turn;
                    *reinterpret_cast<u32x4_t*>(to + ((c * (8 / BITS) + at / 2) ^ f) * 32 + (at & 1) * 16) = v;
                }
            }
        }
        if constexpr (!TRANS)
            if (tid < BJ) Ss[tid] = s_next[0];
    };

    f32x4_t acc[TI][TJ] = {};
    const auto compute = [&] {
        [[maybe_unused]] float scale[TJ];
        [[maybe_unused]] u32x4_t code[TJ];
        if constexpr (!TRANS) {
#pragma unroll
            for (int y = 0; y < TJ; ++y) {
                const int row = wj + 16 * y + li;
                scale[y] = mx_scale((Ss[row] >> (8 * (lk >> 1))) & 0xFFu);
                if constexpr (BITS == 4) {
                    const u32x2_t c = *reinterpret_cast<const u32x2_t*>(Qs + row * kQRow + ((lk >> 1) ^ ((row >> 3) & 1)) * 16 + (lk & 1) * 8);
                    code[y] = u32x4_t{c[0], c[1], 0u, 0u};
                } else {
                    code[y] = *reinterpret_cast<const u32x4_t*>(Qs + row * kQRow + (lk ^ row_group(row)) * 16);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            bf16x8 pv[TI];
#pragma unroll
            for (int x = 0; x < TI; ++x) {
                const int row = wi + 16 * x + li, c = TRANS ? 4 * u + lk : 2 * lk + u;
                if constexpr (PT)
                    pv[x] = transposed(Ps, kPRow, wi / 16 + x, u);
                else
                    pv[x] = *reinterpret_cast<const bf16x8*>(Ps + row * kPRow + (c ^ p_swizzle(row)) * 16);
            }
#pragma unroll
            for (int y = 0; y < TJ; ++y) {
                bf16x8 qv;
                if constexpr (TRANS) {
                    qv = transposed(Qs, kQRow, wj / 16 + y, u);
                } else {
                    u32x4_t d;
                    if constexpr (BITS == 4) {
                        const uint32_t c = code[y][u];
                        d = u32x4_t{mx_pair_bf16<4, 0>(c, scale[y]), mx_pair_bf16<4, 1>(c, scale[y]), mx_pair_bf16<4, 2>(c, scale[y]),
                                    mx_pair_bf16<4, 3>(c, scale[y])};
                    } else {
                        const uint32_t c0 = code[y][2 * u], c1 = code[y][2 * u + 1];
                        d = u32x4_t{mx_pair_bf16<8, 0>(c0, scale[y]), mx_pair_bf16<8, 1>(c0, scale[y]), mx_pair_bf16<8, 0>(c1, scale[y]),
                                    mx_pair_bf16<8, 1>(c1, scale[y])};
                    }
                    qv = __builtin_bit_cast(bf16x8, d);
                }
#pragma unroll
                for (int x = 0; x < TI; ++x)
                    acc[x][y] = YROWS ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(qv, pv[x], acc[x][y], 0, 0, 0)
                                      : __builtin_amdgcn_mfma_f32_16x16x32_bf16(pv[x], qv, acc[x][y], 0, 0, 0);
            }
        }
    };
    const bool whole = place.split < 0;
    float* const sums = g.sums + (whole ? blockIdx.x : g.cut.slots + place.split * g.cut.rest() + place.shared) * (BI * BJ);
    // the lane's place in the tile, computed anew each time: kept, its addresses would take registers from the sums
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
                    store_four<YROWS>(a, n, i0 + ti, j0 + tj, acc[x][y]);
                else
                    *so_far = acc[x][y];
                acc[x][y] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
    };

    int64_t t = t0;
    const int64_t all = g.steps * g.planes, t1 = place.split < 0 ? all : lesser(t + g.cut.per, all);
    if (t < t1) {
        fetch();
        stage();
    }
    for (bool first = true;; first = false) {
        const int64_t end = lesser(t + g.chain, t1);
        for (; t < end; ++t) {
            __syncthreads();
            if (t + 1 < t1) fetch();
            compute();
            __syncthreads();
            if (t + 1 < t1) stage();
        }
        put(first, t >= t1);
        if (t >= t1) break;
    }
}

// A side's eight terms from k on, among steps of all sides (a plane of the workspace).
__device__ __forceinline__ int64_t packed_at(int64_t side, int64_t k, int64_t s) { return (k / kStep * s + side) * kStep + k % kStep; }

// A microscaled X in bf16 (exact), zeros from `terms` on.  A thread takes eight values.
__global__ __launch_bounds__(256) void mx_unpack_kernel(MxMat x, int64_t s, int64_t terms, uint16_t* to, int64_t pieces, int64_t first) {
    const int64_t id = first + blockIdx.x * int64_t(256) + threadIdx.x;
    const int64_t side = id / pieces, k = id % pieces * 8;
    if (side >= s) return;
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    if (k < terms) {   // up to the end of its last block a row's codes are zero
        if (x.bits == 4)
            mx_eight<4>(x.codes + side * x.ldc, x.scales + side * x.lds, k, v);
        else
            mx_eight<8>(x.codes + side * x.ldc, x.scales + side * x.lds, k, v);
    }
    *reinterpret_cast<u32x4_t*>(to + packed_at(side, k, s)) = u32x4_t{v[0], v[1], v[2], v[3]};
}

// X in bf16, zeros from `terms` on.  A workgroup takes 64 sides of a step.
template <bool BF16>
__global__ __launch_bounds__(256) void mx_pack_kernel(const void* X, int64_t ldx, int32_t x_rows, int64_t s, int64_t terms, uint16_t* to,
                                                      int64_t steps, int64_t plane, int64_t first) {
    constexpr int PL = BF16 ? 1 : 3;
    __shared__ uint16_t tile[PL][64][66];
    const int64_t id = first + blockIdx.x, k0 = id % steps * kStep, i0 = id / steps * 64;
    const int lo = threadIdx.x & 63, hi = threadIdx.x >> 6;
    for (int e = 0; e < 16; ++e) {
        // consecutive threads on consecutive elements of X
        const int ti = x_rows ? hi + 4 * e : lo, tk = x_rows ? lo : hi + 4 * e;
        const int64_t i = i0 + ti, k = k0 + tk;
        const bool in = i < s && k < terms;
        const int64_t at = x_rows ? i * ldx + k : k * ldx + i;
        if constexpr (BF16) {
            tile[0][ti][tk] = in ? static_cast<const uint16_t*>(X)[at] : 0;
        } else {
            uint16_t p[3];
            split_bf16(in ? static_cast<const float*>(X)[at] : 0.0f, p);
#pragma unroll
            for (int h = 0; h < 3; ++h) tile[h][ti][tk] = p[h];
        }
    }
    __syncthreads();
    for (int e = 0; e < 16; ++e) {
        const int64_t i = i0 + hi + 4 * e;
        if (i < s)
#pragma unroll
            for (int h = 0; h < PL; ++h) to[h * plane + packed_at(i, k0 + lo, s)] = tile[h][hi + 4 * e][lo];
    }
}

// How a product is cut up.
struct Plan {
    bool pack, by_columns;   // X goes through the workspace; it is taken as it is, a term of every side a row
    int planes;
    int64_t steps, plane, pack_bytes;
    Cut cut;
};

constexpr int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

// x: X and its stride are known (a launch); else the workspace is sized for an X that has to be packed.
Plan make_plan(const MxArgs& a, bool x) {
    Plan p{};
    const int64_t terms = a.trans ? a.q : a.r, n = a.trans ? a.r : a.q;
    p.planes = a.x_bits || a.x_bf16 ? 1 : 3;
    p.steps = ceil_div(terms, kStep);
    p.plane = a.s * p.steps * kStep;
    const uintptr_t at = reinterpret_cast<uintptr_t>(a.X);
    const bool bf16 = x && !a.x_bits && a.x_bf16;
    const bool near = a.ldx < (int64_t(1) << 31) / 256;   // offsets within a tile's rows are 32-bit
    p.by_columns = bf16 && !a.x_rows && near && a.ldx % 2 == 0 && at % 4 == 0;
    p.pack = !p.by_columns && !(bf16 && a.x_rows && near && terms % kStep == 0 && a.ldx % 8 == 0 && at % 16 == 0);
    p.pack_bytes = round_up(p.planes * p.plane * 2, 256);
    p.cut = cut_tiles(a.s, n, p.steps * p.planes, kChain / kStep);
    return p;
}

template <int BITS, bool TRANS, bool PT>
hipError_t launch_tiles(const MxArgs& a, const TileArgs& g, int64_t groups, hipStream_t st) {
    const bool large = g.cut.large;
    const dim3 grid(static_cast<uint32_t>(groups));
    const auto kernel = large ? (a.y_rows ? mx_tile_kernel<BITS, TRANS, PT, 4, 8, true> : mx_tile_kernel<BITS, TRANS, PT, 4, 8, false>)
                              : (a.y_rows ? mx_tile_kernel<BITS, TRANS, PT, 2, 4, true> : mx_tile_kernel<BITS, TRANS, PT, 2, 4, false>);
    kernel<<<grid, kThreads, 0, st>>>(a, g);
    return hipGetLastError();
}

template <int BITS>
hipError_t launch_bits(const MxArgs& a, const TileArgs& g, const Plan& p, int64_t groups, hipStream_t st) {
    if (a.trans) return p.by_columns ? launch_tiles<BITS, true, true>(a, g, groups, st) : launch_tiles<BITS, true, false>(a, g, groups, st);
    return p.by_columns ? launch_tiles<BITS, false, true>(a, g, groups, st) : launch_tiles<BITS, false, false>(a, g, groups, st);
}

}  // namespace

// Offsets within a tile's rows of codes are 32-bit.  Two 4-bit matrices with rows of X further apart than
// mx_scaled_kernel takes go to the general kernel: the workspace is asked for by sizes, and by those that product
// has none for an X in bf16.
bool mx_tiled_serves(const MxArgs& a) {
    const int64_t most = (int64_t(1) << 31) / 256;
    return !(a.x_bits == 4 && a.A.bits == 4) && std::max(a.A.ldc, a.A.lds) < most;
}

int64_t mx_tiled_workspace_bytes(const MxArgs& a) {
    const Plan p = make_plan(a, false);
    return p.pack_bytes + p.cut.sums_bytes();
}

hipError_t launch_mx_tiled(const MxArgs& a, hipStream_t st) {
    const Plan p = make_plan(a, true);
    const int64_t n = a.trans ? a.r : a.q, terms = a.trans ? a.q : a.r;
    TileArgs g{};
    g.P = p.pack ? static_cast<const uint16_t*>(a.workspace) : static_cast<const uint16_t*>(a.X);
    if (p.pack) {
        g.pitch = kStep;
        g.step = a.s * kStep;
        g.extent = a.s * kStep;   // the step's own: what a tile has beyond its sides is not read
        g.shrink = 0;
    } else if (p.by_columns) {
        // With an odd number of sides the last word holds the last side and one element more, which belongs to no
        // side (rows start at words, so it is in the last row's word).
        g.pitch = a.ldx;
        g.step = g.shrink = kStep * a.ldx;
        g.extent = ((terms - 1) * a.ldx + a.s + 1) / 2 * 2;
    } else {
        g.pitch = a.ldx;
        g.step = g.shrink = kStep;
        g.extent = (a.s - 1) * a.ldx + terms;
    }
    g.plane = p.plane;
    g.planes = p.planes;
    g.steps = p.steps;
    g.cut = p.cut;
    g.sums = p.cut.sums_bytes() ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + p.pack_bytes) : nullptr;
    g.chain = chain_steps(a, kStep);
    if (!grid_fits(p.cut.groups(), kThreads)) return hipErrorInvalidConfiguration;
    uint16_t* const packed = static_cast<uint16_t*>(a.workspace);
    constexpr int64_t kMost = int64_t(1) << 20;   // workgroups of a launch: a grid takes sixteen times as many
    if (a.x_bits) {
        const int64_t pieces = p.steps * (kStep / 8), blocks = ceil_div(a.s * pieces, 256);
        for (int64_t b = 0; b < blocks; b += kMost) {
            mx_unpack_kernel<<<dim3(static_cast<uint32_t>(lesser(kMost, blocks - b))), 256, 0, st>>>(a.XM, a.s, terms, packed, pieces, b * 256);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    } else if (p.pack) {
        const auto kernel = a.x_bf16 ? mx_pack_kernel<true> : mx_pack_kernel<false>;
        const int64_t blocks = p.steps * ceil_div(a.s, 64);
        for (int64_t b = 0; b < blocks; b += kMost) {
            kernel<<<dim3(static_cast<uint32_t>(lesser(kMost, blocks - b))), 256, 0, st>>>(a.X, a.ldx, a.x_rows, a.s, terms, packed, p.steps,
                                                                                          p.plane, b);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    const hipError_t e = over_groups(p.cut, [&](int64_t first, int64_t groups) {
        g.first = first;
        return a.A.bits == 4 ? launch_bits<4>(a, g, p, groups, st) : launch_bits<8>(a, g, p, groups, st);
    });
    if (e != hipSuccess || p.cut.splits <= 1) return e;
    return launch_shared_tiles(a, p.cut, g.sums, n, st);
}

}  // namespace coded
