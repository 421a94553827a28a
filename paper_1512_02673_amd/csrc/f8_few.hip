// Products of 8-bit matrices with few right-hand sides: out[i][j] = sum over blocks b of
// sP[b][i] sQ[b][j] (sum over b's columns of P[i][k] Q[j][k]).
//
// Bound: reading Q's codes.  A workgroup takes 16 results, or 32 where that leaves
// two workgroups a compute unit, of all right-hand sides; its four waves take every
// fourth block each and add their sums up in shared memory.  Each wave has a room of
// its own there for three blocks' codes, two of them on their way, in loads of whole
// rows of a block; no wave waits for another.  Codes become bf16 values in
// registers, which is exact, and meet on the bf16 matrix instructions, whose
// products and sums are in fp32, for results of either type.  Where there are few
// workgroups, or more blocks than one chain of additions takes (kF8Chain: 1024 a
// wave), the blocks are split among several, whose sums are joined in order.
//
// Measured, us: 65536 x 8192 times 1 and 16: 93 and 100 (5.8 and 5.4 TB/s; loads in
// the operands' order, half rows, into registers 118 and 126, without non-temporal
// loads 102 and 108, with workgroups in turn instead of runs of them on the XCDs 124
// and 122), 16384 x 4096 times 1 and 32: 13 and 16, 11500 x 5750 times 16: 13.  Small
// tiles (f8_tiled.hip) with up to 64 right-hand sides take 90 (fp32 results 115), 24
// (23) and 22 (28): so from 33 on, or from 17 on where the codes do not stay in the
// memory-side cache.
#include <algorithm>
#include <utility>

#include "f8.h"
#include "to_shared.h"

namespace coded {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kFew = 32, kFewStreamed = 16;   // right-hand sides; where Q's codes do not stay in the memory-side cache

bool streamed(const F8Args& a) { return streams(a.o.q * a.blocks * kF8Block); }

struct FewArgs {
    F8Args a;
    int64_t groups, per, splits;   // workgroups along the results; blocks of a split
    int64_t first;                 // workgroup of this launch among all
    float* part;                   // [split][side][result], or null
};

__device__ __forceinline__ void to_operands(const u32x4_t (&w)[2], bf16x8 (&v)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v[2 * h] = f8_to_bf16(w[h][0], w[h][1]);
        v[2 * h + 1] = f8_to_bf16(w[h][2], w[h][3]);
    }
}

// 8 PE right-hand sides, RT tiles of 16 results.  QB: Q's scales are for 128 rows.  NTL: non-temporal loads of Q.
template <int PE, int RT, bool QB, bool NTL>
__global__ __launch_bounds__(kThreads) void f8_few_kernel(FewArgs g) {
    constexpr int NT = (PE + 1) / 2, kQ = RT * 2048, kStage = kQ + NT * 2048;
    // Three steps of each wave's: three arrays, so that reads of one do not wait for what is on its way into another.
    __shared__ __attribute__((aligned(16))) char step0[4][kStage];
    __shared__ __attribute__((aligned(16))) char step1[4][kStage];
    __shared__ __attribute__((aligned(16))) char step2[4][kStage];
    __shared__ f32x4_t sums[4][NT * RT][64];
    const F8Mat &P = g.a.P, &Q = g.a.Q;
    const MxArgs& o = g.a.o;
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // Workgroups go to the eight XCDs in turn: each takes a run of them.
    const int64_t base = gridDim.x / 8, more = gridDim.x % 8, xcd = blockIdx.x % 8;
    const int64_t id = g.first + xcd * base + lesser(xcd, more) + blockIdx.x / 8, split = id / g.groups;
    const int64_t j0 = id % g.groups * 16 * RT, n = o.q;
    const int s = static_cast<int>(o.s);
    // Load l of a matrix takes rows 8 l .. 8 l + 7, whole blocks of 128 bytes; pieces of 16 bytes lie exchanged by
    // (row >> 1) & 7.  Rows past the last one repeat it, and are not stored.
    uint32_t q_from[2 * RT], p_from[PE], qs[RT][4], ps[NT];
#pragma unroll
    for (int l = 0; l < 2 * RT; ++l) {
        const int row = 8 * l + (lane >> 3);
        q_from[l] = static_cast<uint32_t>(lesser(row, n - 1 - j0) * Q.ldc) + ((lane ^ (row >> 1)) & 7) * 16;
    }
#pragma unroll
    for (int l = 0; l < PE; ++l) {
        const int row = 8 * l + (lane >> 3);
        p_from[l] = static_cast<uint32_t>(lesser(row, s - 1) * P.ldc) + ((lane ^ (row >> 1)) & 7) * 16;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) qs[r][e] = 4 * static_cast<uint32_t>(lesser(16 * r + 4 * lk + e, n - 1 - j0));
#pragma unroll
    for (int t = 0; t < NT; ++t) ps[t] = 4 * static_cast<uint32_t>(lesser(16 * t + li, s - 1) >> (P.block_rows == 1 ? 0 : 7));

    f32x4_t acc[RT][NT] = {};
    const int64_t b0 = split * g.per + wave, b1 = lesser((split + 1) * g.per, g.a.blocks);
    const int64_t steps = b0 < b1 ? ceil_div(b1 - b0, 4) : 0;   // this wave's: every fourth block
    struct Scales {
        f32x4_t q[RT];
        float p[NT];
    };
    const auto load = [&](char* to, Scales& f, int64_t k) {
        const bool there = k < steps;
        const int64_t at = b0 + 4 * (there ? k : steps - 1);   // past the last step: that one again, times zero
        const Window q(Q.codes + j0 * Q.ldc + at * kF8Block, 0xFFFFFFFF), p(P.codes + at * kF8Block, 0xFFFFFFFF);
#pragma unroll
        for (int l = 0; l < 2 * RT; ++l) sixteen_to_shared<NTL>(q, to + l * 1024, q_from[l]);
#pragma unroll
        for (int l = 0; l < PE; ++l) sixteen_to_shared(p, to + kQ + l * 1024, p_from[l]);
        const Window sp(P.scales + at * P.lds, 0xFFFFFFFF);
#pragma unroll
        for (int t = 0; t < NT; ++t) f.p[t] = there ? __uint_as_float(sp.word(ps[t])) : 0.0f;
        if constexpr (QB) {
            const float one = Q.scales[at * Q.lds + (j0 >> 7)];
#pragma unroll
            for (int r = 0; r < RT; ++r) f.q[r] = f32x4_t{one, one, one, one};
        } else {
            const Window sq(Q.scales + at * Q.lds + j0, 0xFFFFFFFF);
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) f.q[r][e] = __uint_as_float(sq.word(qs[r][e]));
        }
    };
    const auto operands = [&](const char* tile, bf16x8 (&v)[4]) {
        u32x4_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = *reinterpret_cast<const u32x4_t*>(tile + li * 128 + (((lk + 4 * h) ^ (li >> 1)) & 7) * 16);
        to_operands(w, v);
    };
    const auto multiply = [&](const char* from, const Scales& f) {
        bf16x8 qv[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) operands(from + r * 2048, qv[r]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bf16x8 pv[4];
            operands(from + kQ + t * 2048, pv);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 4; ++k) v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qv[r][k], pv[k], v, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[r][t][e] = fmaf(v[e], f.p[t] * f.q[r][e], acc[r][t][e]);
            }
        }
        // what was read is here before its place is loaded again
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
        Scales f0, f1, f2;
        load(step0[wave], f0, 0);
        load(step1[wave], f1, 1);
        for (int64_t k = 0; k < steps; k += 3) {
            load(step2[wave], f2, k + 2);
            multiply(step0[wave], f0);
            load(step0[wave], f0, k + 3);
            multiply(step1[wave], f1);
            load(step1[wave], f1, k + 4);
            multiply(step2[wave], f2);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // shared memory is another workgroup's after this one
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) sums[wave][r * NT + t][lane] = acc[r][t];
    __syncthreads();
    // a result a thread: those of one right-hand side next to each other
    for (int k = tid; k < 16 * RT * s; k += kThreads) {
        const int j = k % (16 * RT), i = k / (16 * RT);
        const int at = j / 16 * NT + i / 16, from = (i % 16 + j % 16 / 4 * 16) * 4 + j % 4;
        const float* const one = reinterpret_cast<const float*>(sums) + at * 256 + from;
        float v = one[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) v += one[w * NT * RT * 256];
        if (j0 + j >= n) continue;
        if (g.part)
            g.part[(split * s + i) * n + j0 + j] = v;
        else
            mx_store(o, i, j0 + j, v);
    }
}

struct Plan {
    int rt;
    int64_t groups, per, splits;
};
Plan plan_of(const F8Args& a) {
    Plan p{};
    p.rt = ceil_div(a.o.q, 32) >= 512 ? 2 : 1;
    p.groups = ceil_div(a.o.q, 16 * p.rt);
    const int64_t few = std::min(ceil_div(a.blocks, 8), 512 / std::max<int64_t>(1, p.groups));
    const int64_t splits = std::max<int64_t>(1, std::max(few, ceil_div(a.blocks, kF8Chain)));
    p.per = std::max<int64_t>(1, ceil_div(a.blocks, splits));
    p.splits = std::max<int64_t>(1, ceil_div(a.blocks, p.per));
    return p;
}

template <int PE, int RT>
hipError_t launch_one(const FewArgs& g, int64_t groups, hipStream_t st) {
    const bool blocked = g.a.Q.block_rows != 1;
    auto kernel = blocked ? f8_few_kernel<PE, RT, true, false> : f8_few_kernel<PE, RT, false, false>;
    if constexpr (8 * PE <= kFewStreamed)   // more right-hand sides of a streamed matrix are the tiles'
        if (streamed(g.a)) kernel = blocked ? f8_few_kernel<PE, RT, true, true> : f8_few_kernel<PE, RT, false, true>;
    kernel<<<dim3(static_cast<uint32_t>(groups)), kThreads, 0, st>>>(g);
    return hipGetLastError();
}

template <int PE>
hipError_t launch_rows(const FewArgs& g, int rt, int64_t groups, hipStream_t st) {
    return rt == 2 ? launch_one<PE, 2>(g, groups, st) : launch_one<PE, 1>(g, groups, st);
}

}  // namespace

bool f8_few_serves(const F8Args& a) { return a.o.s <= (streamed(a) ? kFewStreamed : kFew); }

int64_t f8_few_workspace_bytes(const F8Args& a) {
    const Plan p = plan_of(a);
    return p.splits > 1 ? p.splits * a.o.s * a.o.q * 4 : 0;
}

hipError_t launch_f8_few(const F8Args& a, hipStream_t st) {
    const Plan p = plan_of(a);
    FewArgs g{a, p.groups, p.per, p.splits, 0, p.splits > 1 ? static_cast<float*>(a.o.workspace) : nullptr};
    const int64_t all = p.groups * p.splits, most = int64_t(1) << 23;
    for (; g.first < all; g.first += most) {
        const int64_t groups = lesser(most, all - g.first);
        const hipError_t e = a.o.s <= 8 ? launch_rows<1>(g, p.rt, groups, st) : a.o.s <= 16 ? launch_rows<2>(g, p.rt, groups, st) : launch_rows<4>(g, p.rt, groups, st);
        if (e != hipSuccess) return e;
    }
    return p.splits > 1 ? launch_mx_join(a.o, g.part, p.splits, a.o.q, st) : hipSuccess;
}

// The sides change places where few results of many right-hand sides are few right-hand sides with many results, and
// where Y has the other order: the tiles write rows of it.
static F8Args arranged(F8Args a) {
    if (f8_few_serves(a)) return a;
    F8Args other = a;
    std::swap(other.P, other.Q);
    std::swap(other.o.q, other.o.s);
    other.o.y_rows = !a.o.y_rows;
    return f8_few_serves(other) || !a.o.y_rows ? other : a;
}

int64_t f8_workspace_bytes(const F8Args& given) {
    const F8Args a = arranged(given);
    return f8_few_serves(a) ? f8_few_workspace_bytes(a) : f8_tiled_workspace_bytes(a);
}

hipError_t launch_f8_product(F8Args given, hipStream_t st) {
    const F8Args a = arranged(given);
    return f8_few_serves(a) ? launch_f8_few(a, st) : launch_f8_tiled(a, st);
}

}  // namespace coded
