// Products of 8-bit matrices, results 16 rows of Q at a time: out[i][j] = sum over
// blocks b of sP[b][i] sQ[b][j] (sum over b's columns of P[i][k] Q[j][k]).
//
// Codes become bf16 values in registers, which is exact, and meet on the bf16
// matrix instructions, whose products and sums are in fp32.  A workgroup takes 16
// results of 16 NT right-hand sides; its four waves take blocks in turn and add
// their sums up in shared memory.  Lane (li, lk) of a block holds columns 16 lk ..
// 16 lk + 15 and 64 more of row li, so a load takes 64 bytes of each row.
// Where there are few workgroups the blocks are split among several, whose sums
// are joined in order.
#include <algorithm>
#include <utility>

#include "f8.h"

namespace coded {
namespace {

constexpr int kThreads = 256;

struct FewArgs {
    F8Args a;
    int64_t groups_j, groups_i, per, splits;   // workgroups along the results and the right-hand sides; blocks of a split
    int64_t first;                             // workgroup of this launch among all
    float* part;                               // [split][side][result], or null
};

__device__ __forceinline__ void load_block(const uint8_t* row, int lk, u32x4_t (&w)[2]) {
    w[0] = *reinterpret_cast<const u32x4_t*>(row + 16 * lk);
    w[1] = *reinterpret_cast<const u32x4_t*>(row + 64 + 16 * lk);
}
__device__ __forceinline__ void to_operands(const u32x4_t (&w)[2], bf16x8 (&v)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v[2 * h] = f8_to_bf16(w[h][0], w[h][1]);
        v[2 * h + 1] = f8_to_bf16(w[h][2], w[h][3]);
    }
}

template <int NT>
__global__ __launch_bounds__(kThreads) void f8_few_kernel(FewArgs g) {
    __shared__ f32x4_t sums[4][NT][64];
    const F8Mat P = g.a.P, Q = g.a.Q;
    const MxArgs& o = g.a.o;
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t id = g.first + blockIdx.x, gj = id % g.groups_j, gi = id / g.groups_j % g.groups_i, split = id / g.groups_j / g.groups_i;
    const int64_t j0 = gj * 16, i0 = gi * 16 * NT, n = o.q, s = o.s;
    // rows past the last one repeat it, and are not stored
    const uint8_t* qrow = Q.codes + lesser(j0 + li, n - 1) * Q.ldc;
    int64_t qs[4];
    const uint8_t* prow[NT];
    int64_t ps[NT];
#pragma unroll
    for (int e = 0; e < 4; ++e) qs[e] = lesser(j0 + 4 * lk + e, n - 1) / Q.block_rows;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t i = lesser(i0 + 16 * t + li, s - 1);
        prow[t] = P.codes + i * P.ldc;
        ps[t] = i / P.block_rows;
    }
    f32x4_t acc[NT] = {};
    const int64_t b1 = lesser((split + 1) * g.per, g.a.blocks);
    for (int64_t b = split * g.per + wave; b < b1; b += 4) {
        u32x4_t w[2];
        bf16x8 qv[4];
        load_block(qrow + b * kF8Block, lk, w);
        to_operands(w, qv);
        float sq[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sq[e] = Q.scales[b * Q.lds + qs[e]];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            u32x4_t x[2];
            bf16x8 pv[4];
            load_block(prow[t] + b * kF8Block, lk, x);
            to_operands(x, pv);
            const float sp = P.scales[b * P.lds + ps[t]];
            f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 4; ++u) v = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qv[u], pv[u], v, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][e] = fmaf(v[e], sp * sq[e], acc[t][e]);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < NT; t += 4) {
        f32x4_t v = sums[0][t][lane];
#pragma unroll
        for (int k = 1; k < 4; ++k) v += sums[k][t][lane];
        const int64_t i = i0 + 16 * t + li;
        if (i >= s) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t j = j0 + 4 * lk + e;
            if (j >= n) break;
            if (g.part)
                g.part[(split * s + i) * n + j] = v[e];
            else
                mx_store(o, i, j, v[e]);
        }
    }
}

struct Plan {
    int nt;
    int64_t groups_j, groups_i, per, splits;
};
Plan plan_of(const F8Args& a) {
    Plan p{};
    p.nt = a.o.s <= 16 ? 1 : a.o.s <= 32 ? 2 : 4;
    p.groups_j = ceil_div(a.o.q, 16);
    p.groups_i = ceil_div(a.o.s, 16 * p.nt);
    const int64_t groups = p.groups_j * p.groups_i;
    const int64_t splits = std::max<int64_t>(1, std::min(ceil_div(a.blocks, 8), 1024 / std::max<int64_t>(1, groups)));
    p.per = std::max<int64_t>(1, ceil_div(a.blocks, splits));
    p.splits = std::max<int64_t>(1, ceil_div(a.blocks, p.per));
    return p;
}

}  // namespace

bool f8_few_serves(const F8Args& a) { return a.o.s <= 64; }

int64_t f8_few_workspace_bytes(const F8Args& a) {
    const Plan p = plan_of(a);
    return p.splits > 1 ? p.splits * a.o.s * a.o.q * 4 : 0;
}

hipError_t launch_f8_few(const F8Args& a, hipStream_t st) {
    const Plan p = plan_of(a);
    FewArgs g{a, p.groups_j, p.groups_i, p.per, p.splits, 0, p.splits > 1 ? static_cast<float*>(a.o.workspace) : nullptr};
    const int64_t all = p.groups_j * p.groups_i * p.splits, most = int64_t(1) << 23;
    const auto kernel = p.nt == 1 ? f8_few_kernel<1> : p.nt == 2 ? f8_few_kernel<2> : f8_few_kernel<4>;
    for (; g.first < all; g.first += most) {
        kernel<<<dim3(static_cast<uint32_t>(lesser(most, all - g.first))), kThreads, 0, st>>>(g);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return p.splits > 1 ? launch_mx_join(a.o, g.part, p.splits, a.o.q, st) : hipSuccess;
}

// The sides change places where Y has the other order: the tiles write rows of it, and few results of many
// right-hand sides are few right-hand sides with many results.
static F8Args arranged(F8Args a) {
    const bool turn = f8_few_serves(a) ? false : a.o.q <= 64 ? true : !a.o.y_rows;
    if (turn) {
        std::swap(a.P, a.Q);
        std::swap(a.o.q, a.o.s);
        a.o.y_rows = !a.o.y_rows;
    }
    return a;
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
