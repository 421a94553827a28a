// Rows of a table by tokens, and the gradient of the table.
//
// The gradient sorts the tokens with their places (stably) and then adds up runs of equal tokens.  Up to kSmall
// tokens a token's place is the number of those before it, counted; more are
// sorted digit by digit.  The sorted places are cut into chunks; a workgroup adds
// up a chunk's rows and writes the sums of the runs that lie in it.  A run that
// goes on in the next chunk leaves its part of the sum in the workspace, and
// embed_join_kernel adds these up.  Nothing is added by atomics, so the sums
// depend on the tokens alone.
//
// Bound: memory.  Measured, 65536 tokens, 4096 columns, a table of 65536 rows: the lookup (bf16)
// 180 to 200 us (0.5 GB written, rows of 16940 tokens read), the gradient (bf16 rows, fp32 table of
// which 1.07 GB are written) 396: sorting 35, sums and zeros 324 (4.9 TB/s), joining 28, as the most
// frequent token's 4131 rows make one run.  1000 tokens, 512 columns, 16384 rows of fp32: 3, and 5 + 10 + 4.
// Workgroups that write zeros first took 20 us more, mixed among the others 110; places looked up only
// when their rows were wanted 34.
#include <algorithm>

#include "layers.h"

namespace coded {
namespace {

constexpr int kThreads = 256, kLogThreads = 8;
constexpr int kSmall = 4096;     // tokens that are sorted by counting
constexpr int kMostBins = 512, kMostBlocks = 256;

// A token's row; `vocab` for one that has none.
template <bool WIDE>
__device__ __forceinline__ uint32_t row_of(const void* tok, int64_t i, int64_t vocab, int64_t skip) {
    const int64_t t = WIDE ? static_cast<const int64_t*>(tok)[i] : static_cast<int64_t>(static_cast<const int32_t*>(tok)[i]);
    return t < 0 || t >= vocab || t == skip ? static_cast<uint32_t>(vocab) : static_cast<uint32_t>(t);
}

template <bool WIDE, bool E16, bool O16>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a, RowCut cut) {
    const int64_t i = blockIdx.x / cut.pieces * cut.rows(kThreads) + (threadIdx.x >> cut.log_tpr);
    const int64_t c = ((blockIdx.x % cut.pieces << cut.log_tpr) + (threadIdx.x & ((1 << cut.log_tpr) - 1))) * 8;
    if (i >= a.n || c >= a.d) return;
    const int64_t t = WIDE ? static_cast<const int64_t*>(a.tok)[i] : static_cast<int64_t>(static_cast<const int32_t*>(a.tok)[i]);
    float v[8];
    if (t != a.skip && t >= 0 && t < a.vocab) {
        row_load<E16>(static_cast<const char*>(a.E) + t * a.lde * (E16 ? 2 : 4), c, a.d, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= a.scale;
    } else {   // a token that the table lacks is NaN, also where skip is that number
        const float none = t >= 0 && t < a.vocab ? 0.0f : __builtin_nanf("");
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = none;
    }
    row_store<O16>(static_cast<char*>(a.out) + i * a.ldo * (O16 ? 2 : 4), c, a.d, v);
}

// ---------------------------------------------------------------- sorting

// Token i's place is the number of tokens with a lower row, and of earlier ones with the same.  A workgroup places
// 64 tokens; each of its sixteen waves compares them with a sixteenth of all.  1000 tokens: 5.4 us, with four waves
// 9.3; lookup and gradient on an idle card 47 and 51, and 27 both ways where calls queue and the host bounds them.
constexpr int kCountWaves = 16;
template <bool WIDE>
__global__ __launch_bounds__(kCountWaves * 64) void embed_count_kernel(const void* tok, int n, int64_t vocab, int64_t skip, uint32_t* keys,
                                                                     uint32_t* index) {
    __shared__ __attribute__((aligned(16))) uint32_t all[kSmall];
    __shared__ int before[kCountWaves][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (n + 4 * kCountWaves - 1) / (4 * kCountWaves) * 4;   // of all, a wave's: whole pieces of 16 bytes
    for (int i = tid; i < each * kCountWaves; i += kCountWaves * 64) all[i] = i < n ? row_of<WIDE>(tok, i, vocab, skip) : 0xFFFFFFFFu;
    __syncthreads();
    const int i = blockIdx.x * 64 + lane;
    const uint32_t mine = i < n ? all[i] : 0u;
    int count = 0;
    for (int j = wave * each; j < (wave + 1) * each; j += 4) {
        const u32x4_t k = *reinterpret_cast<const u32x4_t*>(all + j);
#pragma unroll
        for (int e = 0; e < 4; ++e) count += k[e] < mine + (j + e < i ? 1u : 0u);
    }
    before[wave][lane] = count;
    __syncthreads();
    if (wave == 0 && i < n) {
        int at = 0;
#pragma unroll
        for (int w = 0; w < kCountWaves; ++w) at += before[w][lane];
        keys[at] = mine;
        index[at] = static_cast<uint32_t>(i);
    }
}

// One digit of a sort: `bins` values of (key >> shift); a workgroup takes `per` keys (a multiple of 256).
struct Digit {
    int64_t n, per;
    int shift, bits, blocks;
};

template <bool FIRST, bool WIDE>
__device__ __forceinline__ uint32_t key_at(const void* from, int64_t i, int64_t vocab, int64_t skip) {
    if constexpr (FIRST)
        return row_of<WIDE>(from, i, vocab, skip);
    else
        return static_cast<const uint32_t*>(from)[i];
}

// counts[block][value of the digit]
template <bool FIRST, bool WIDE>
__global__ __launch_bounds__(kThreads) void embed_digits_kernel(const void* from, int64_t vocab, int64_t skip, Digit d, uint32_t* counts) {
    __shared__ uint32_t bin[kMostBins];
    const int bins = 1 << d.bits;
    for (int b = threadIdx.x; b < bins; b += kThreads) bin[b] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * d.per, end = lesser(first + d.per, d.n);
    for (int64_t i = first + threadIdx.x; i < end; i += kThreads)
        atomicAdd(&bin[(key_at<FIRST, WIDE>(from, i, vocab, skip) >> d.shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) counts[blockIdx.x * bins + b] = bin[b];
}

// Each key to its place by this digit, keys of one value in the order they had.  Waves take consecutive quarters of the
// workgroup's keys, 64 keys at a time; keys of one value find each other by one vote a bit.
template <bool FIRST, bool WIDE>
__global__ __launch_bounds__(kThreads) void embed_place_kernel(const void* from, const uint32_t* index, int64_t vocab, int64_t skip, Digit d,
                                                              const uint32_t* counts, uint32_t* keys_out, uint32_t* index_out) {
    __shared__ uint32_t next[4][kMostBins];    // where a wave's next key of a value goes
    __shared__ uint32_t total[kThreads];
    const int bins = 1 << d.bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = blockIdx.x * d.per, quarter = d.per / 4;
    const int64_t w0 = lesser(first + wave * quarter, d.n), w1 = lesser(w0 + quarter, d.n);
    for (int b = lane; b < bins; b += 64) next[wave][b] = 0;
    __syncthreads();
    for (int64_t i = w0 + lane; i < w1; i += 64)
        atomicAdd(&next[wave][(key_at<FIRST, WIDE>(from, i, vocab, skip) >> d.shift) & (bins - 1)], 1u);
    // two consecutive values a thread: how many keys have them, in all workgroups and in those before this one
    uint32_t sum[2] = {0, 0}, before[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int b = 2 * tid + h;
        if (b >= bins) continue;
#pragma unroll 8
        for (int k = 0; k < d.blocks; ++k) {
            const uint32_t c = counts[k * bins + b];
            sum[h] += c;
            before[h] += k < static_cast<int>(blockIdx.x) ? c : 0u;
        }
    }
    total[tid] = sum[0] + sum[1];
    __syncthreads();
    for (int step = 1; step < kThreads; step *= 2) {
        const uint32_t v = tid >= step ? total[tid - step] : 0u;
        __syncthreads();
        total[tid] += v;
        __syncthreads();
    }
    uint32_t base = total[tid] - sum[0] - sum[1];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int b = 2 * tid + h;
        if (b >= bins) continue;
        uint32_t at = base + before[h];
        for (int w = 0; w < 4; ++w) {
            const uint32_t c = next[w][b];
            next[w][b] = at;
            at += c;
        }
        base += sum[h];
    }
    __syncthreads();
    for (int64_t i = w0; i < w1; i += 64) {
        const bool in = i + lane < w1;
        const uint32_t key = in ? key_at<FIRST, WIDE>(from, i + lane, vocab, skip) : 0u;
        const uint32_t value = (key >> d.shift) & (bins - 1);
        uint64_t same = __ballot(in);
        for (int b = 0; b < d.bits; ++b) {
            const bool bit = (value >> b) & 1;
            const uint64_t v = __ballot(bit);
            same &= bit ? v : ~v;
        }
        const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
        if (in) {
            const uint32_t at = next[wave][value] + rank;
            keys_out[at] = key;
            index_out[at] = FIRST ? static_cast<uint32_t>(i + lane) : index[i + lane];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the reads above, then the writes, then the next reads
        if (in && rank == 0) next[wave][value] += static_cast<uint32_t>(__popcll(same));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// ---------------------------------------------------------------- sums

// How sorted places are cut into chunks.
struct RunChunks {
    int64_t n, per, count;
    int64_t fill_rows, fills;   // rows of the table that a filling workgroup looks at, and how many there are
};

// Places of keys below (or up to, with UP) `key` in the sorted keys.
template <bool UP>
__device__ __forceinline__ int64_t bound(const uint32_t* keys, int64_t n, uint32_t key) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (UP ? keys[mid] <= key : keys[mid] < key)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

template <bool E16>
__device__ __forceinline__ void put_row(const EmbedGradArgs& a, int64_t row, int64_t c, float (&v)[8]) {
    char* to = static_cast<char*>(a.dE) + row * a.ldde * (E16 ? 2 : 4);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= a.scale;
    if (a.beta != 0.0f) {
        float old[8];
        row_load<E16>(to, c, a.d, old);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = fmaf(a.beta, old[k], v[k]);
    }
    row_store<E16>(to, c, a.d, v);
}

// Rows without a token: zero, or beta times what they were.
template <bool E16>
__device__ __forceinline__ void fill_rows(const EmbedGradArgs& a, const uint32_t* keys, const RunChunks& g, const RowCut& cut, int64_t first) {
    __shared__ uint32_t there[kThreads];
    const int tid = threadIdx.x;
    if (tid < g.fill_rows) {
        const uint32_t row = static_cast<uint32_t>(first + tid);
        const int64_t at = first + tid < a.vocab ? bound<false>(keys, g.n, row) : g.n;
        there[tid] = first + tid >= a.vocab || (at < g.n && keys[at] == row);
    }
    __syncthreads();
    constexpr int kSize = E16 ? 2 : 4, kEach = 16 / kSize;
    if (a.beta == 0.0f) {   // 16 bytes a lane, lanes next to each other
        const int lane = tid & 63;
        for (int64_t k = tid >> 6; k < g.fill_rows; k += kThreads / 64) {
            if (there[k]) continue;
            char* const to = static_cast<char*>(a.dE) + (first + k) * a.ldde * kSize;
            const int64_t whole = a.d / kEach;
            for (int64_t c = lane; c < whole; c += 64) *reinterpret_cast<u32x4_bf*>(to + c * 16) = u32x4_t{0u, 0u, 0u, 0u};
            for (int64_t c = whole * kEach + lane; c < a.d; c += 64) {
                if constexpr (E16)
                    reinterpret_cast<uint16_t*>(to)[c] = 0;
                else
                    reinterpret_cast<float*>(to)[c] = 0.0f;
            }
        }
        return;
    }
    const int64_t c0 = (tid & ((1 << cut.log_tpr) - 1)) * 8;
    for (int64_t k = tid >> cut.log_tpr; k < g.fill_rows; k += cut.rows(kThreads)) {
        if (there[k]) continue;
        for (int64_t c = c0; c < a.d; c += int64_t(8) << cut.log_tpr) {
            float v[8] = {};
            put_row<E16>(a, first + k, c, v);
        }
    }
}

__device__ __forceinline__ float* part_of(float* parts, int64_t chunk, int which, int64_t d) { return parts + (chunk * 2 + which) * d; }

template <bool G16, bool E16>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedGradArgs a, const uint32_t* keys, const uint32_t* index, RunChunks g, RowCut cut,
                                                            float* parts) {
    const int64_t id = blockIdx.x, sums = gridDim.x - g.fills;
    if (id >= sums) {
        fill_rows<E16>(a, keys, g, cut, (id - sums) * g.fill_rows);
        return;
    }
    const int64_t chunk = id / cut.pieces * cut.rows(kThreads) + (threadIdx.x >> cut.log_tpr);
    const int64_t c = ((id % cut.pieces << cut.log_tpr) + (threadIdx.x & ((1 << cut.log_tpr) - 1))) * 8;
    if (chunk >= g.count || c >= a.d) return;
    const int64_t p0 = chunk * g.per, p1 = lesser(p0 + g.per, g.n);
    const uint32_t none = static_cast<uint32_t>(a.vocab);
    uint32_t run = keys[p0];
    bool head = p0 > 0 && keys[p0 - 1] == run;      // the run began in a chunk before
    float sum[8] = {};
    const auto end_run = [&](bool tail) {           // tail: it goes on in the next one
        if (run != none) {
            if (head || tail)
                row_store<false>(part_of(parts, chunk, head ? 0 : 1, a.d), c, a.d, sum);
            else
                put_row<E16>(a, run, c, sum);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
        head = false;
    };
    // Rows in groups of kRows at once, and the next group's keys and places meanwhile; past the end the last one again.
    constexpr int kRows = G16 ? 8 : 4;
    uint32_t key[kRows], place[kRows];
    const auto look = [&](int64_t p) {
#pragma unroll
        for (int e = 0; e < kRows; ++e) {
            const int64_t at = lesser(p + e, p1 - 1);
            key[e] = keys[at];
            place[e] = index[at];
        }
    };
    look(p0);
    for (int64_t p = p0; p < p1; p += kRows) {
        float v[kRows][8];
        uint32_t now[kRows];
#pragma unroll
        for (int e = 0; e < kRows; ++e) {
            now[e] = key[e];
            row_load<G16>(static_cast<const char*>(a.G) + static_cast<int64_t>(place[e]) * a.ldg * (G16 ? 2 : 4), c, a.d, v[e]);
        }
        look(p + kRows);
#pragma unroll
        for (int e = 0; e < kRows; ++e) {
            if (p + e >= p1) break;
            if (now[e] != run) {
                end_run(false);
                run = now[e];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum[k] += v[e][k];
        }
    }
    end_run(p1 < g.n && keys[p1] == run);
}

// The sums of the runs that begin in a chunk and go on in the next.  A workgroup takes 512 columns of one chunk's; its
// four waves take parts in turn, and add up kMostParts of them, then such sums: at 2^31 tokens a chunk has 2048 rows, and a
// chain of additions is at most 2048, 513 or 512 long, not the 2^18 of a wave's parts one after another.
constexpr int kMostParts = 512;
template <bool E16>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(EmbedGradArgs a, const uint32_t* keys, RunChunks g, int64_t pieces, float* parts) {
    __shared__ float sums[4][64][9];
    const int64_t chunk = blockIdx.x / pieces;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (blockIdx.x % pieces * 64 + lane) * 8;
    const int64_t p0 = chunk * g.per, p1 = p0 + g.per;
    if (p1 >= g.n) return;      // the same for the whole workgroup, as the next lines are
    const uint32_t run = keys[p1];
    if (run == static_cast<uint32_t>(a.vocab) || keys[p1 - 1] != run || (p0 > 0 && keys[p0 - 1] == run)) return;
    const int64_t last = (bound<true>(keys, g.n, run) - 1) / g.per;     // the chunk in which the run ends
    float sum[8] = {};
    if (c < a.d) {
        if (wave == 0) row_load<false>(part_of(parts, chunk, 1, a.d), c, a.d, sum);
        const float* from = part_of(parts, chunk + 1 + wave, 0, a.d);
        int left = static_cast<int>((last - chunk - wave + 3) / 4);   // every fourth part
        const auto add_some = [&] {
            const int some = left < kMostParts ? left : kMostParts;
            left -= some;
#pragma unroll 8
            for (int k = 0; k < some; ++k) {
                float v[8];
                row_load<false>(from, c, a.d, v);
                from += 8 * a.d;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += v[e];
            }
        };
        add_some();
        if (left > 0) {
            float* const all = sums[wave][lane];    // in shared memory: the loop needs the registers
#pragma unroll
            for (int e = 0; e < 8; ++e) all[e] = sum[e];
            while (left > 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
                add_some();
#pragma unroll
                for (int e = 0; e < 8; ++e) all[e] += sum[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = all[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][lane][e] = sum[e];
    __syncthreads();
    if (wave != 0 || c >= a.d) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = (sum[e] + sums[1][lane][e]) + (sums[2][lane][e] + sums[3][lane][e]);
    put_row<E16>(a, run, c, sum);
}

constexpr int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

// What the workspace holds: two sets of keys and places, the digits' counts, the parts of sums.
struct Plan {
    int64_t n, list, parts;
    RunChunks chunks;
    RowCut cut;
    int64_t bytes() const { return 4 * list + kMostBlocks * kMostBins * 4 + parts; }
};
Plan plan_of(int64_t n, int64_t vocab, int64_t d) {
    Plan p{};
    p.n = n;
    p.cut = cut_rows(d, kLogThreads);
    p.list = round_up(n * 4, 256);
    p.chunks.n = n;
    p.chunks.per = std::max(std::min<int64_t>(64, std::max<int64_t>(8, n / 1024)), ceil_div(n, int64_t(1) << 20));
    p.chunks.count = ceil_div(n, p.chunks.per);
    p.parts = round_up(p.chunks.count * 2 * d * 4, 256);
    return p;
}

template <bool WIDE>
hipError_t sort_tokens(const EmbedGradArgs& a, const Plan& p, uint32_t*& keys, uint32_t*& index, hipStream_t st) {
    char* const ws = static_cast<char*>(a.workspace);
    uint32_t* k[2] = {reinterpret_cast<uint32_t*>(ws), reinterpret_cast<uint32_t*>(ws + 2 * p.list)};
    uint32_t* x[2] = {reinterpret_cast<uint32_t*>(ws + p.list), reinterpret_cast<uint32_t*>(ws + 3 * p.list)};
    keys = k[0];
    index = x[0];
    if (a.n <= kSmall) {
        embed_count_kernel<WIDE><<<dim3(static_cast<uint32_t>(ceil_div(a.n, 64))), kCountWaves * 64, 0, st>>>(a.tok, static_cast<int>(a.n), a.vocab, a.skip, keys, index);
        return hipGetLastError();
    }
    uint32_t* counts = reinterpret_cast<uint32_t*>(ws + 4 * p.list);
    int bits = 1;
    while (a.vocab >> bits) ++bits;   // keys are 0 .. vocab
    const int passes = static_cast<int>(ceil_div(bits, 9));
    Digit d{};
    d.n = a.n;
    d.per = std::max<int64_t>(1024, round_up(ceil_div(a.n, kMostBlocks), 256));
    d.blocks = static_cast<int>(ceil_div(a.n, d.per));
    const dim3 grid(static_cast<uint32_t>(d.blocks));
    for (int pass = 0; pass < passes; ++pass) {
        d.shift = bits * pass / passes;
        d.bits = bits * (pass + 1) / passes - d.shift;
        const int to = pass & 1;
        if (pass == 0) {
            embed_digits_kernel<true, WIDE><<<grid, kThreads, 0, st>>>(a.tok, a.vocab, a.skip, d, counts);
            embed_place_kernel<true, WIDE><<<grid, kThreads, 0, st>>>(a.tok, nullptr, a.vocab, a.skip, d, counts, k[to], x[to]);
        } else {
            embed_digits_kernel<false, WIDE><<<grid, kThreads, 0, st>>>(keys, a.vocab, a.skip, d, counts);
            embed_place_kernel<false, WIDE><<<grid, kThreads, 0, st>>>(keys, index, a.vocab, a.skip, d, counts, k[to], x[to]);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        keys = k[to];
        index = x[to];
    }
    return hipSuccess;
}

// Workgroups of the sums, of the joins, and table rows that a workgroup fills.
int64_t sum_blocks(const Plan& p) { return ceil_div(p.chunks.count, p.cut.rows(kThreads)) * p.cut.pieces; }
int64_t join_pieces(int64_t d) { return ceil_div(d, 512); }
int64_t join_blocks(const Plan& p, int64_t d) { return std::max<int64_t>(0, p.chunks.count - 1) * join_pieces(d); }
int64_t fill_rows(int64_t vocab) { return std::min<int64_t>(kThreads, std::max<int64_t>(1, vocab / 2048)); }

template <bool G16, bool E16>
hipError_t sum_rows(const EmbedGradArgs& a, Plan p, const uint32_t* keys, const uint32_t* index, hipStream_t st) {
    float* parts = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + 4 * p.list + kMostBlocks * kMostBins * 4);
    RunChunks& g = p.chunks;
    if (a.beta != 1.0f) {
        g.fill_rows = fill_rows(a.vocab);
        g.fills = ceil_div(a.vocab, g.fill_rows);
    }
    const int64_t blocks = g.fills + sum_blocks(p);
    if (blocks == 0) return hipSuccess;
    embed_sum_kernel<G16, E16><<<dim3(static_cast<uint32_t>(blocks)), kThreads, 0, st>>>(a, keys, index, g, p.cut, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.count < 2) return e;
    embed_join_kernel<E16><<<dim3(static_cast<uint32_t>(join_blocks(p, a.d))), kThreads, 0, st>>>(a, keys, g, join_pieces(a.d), parts);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
    const RowCut cut = cut_rows(a.d, kLogThreads);
    const int64_t step = (int64_t(1) << 23) / cut.pieces * cut.rows(kThreads);
    if (step < 1) return hipErrorInvalidConfiguration;
    for (int64_t at = 0; at < a.n; at += step) {
        EmbedArgs p = a;
        p.n = lesser(step, a.n - at);
        p.tok = static_cast<const char*>(a.tok) + at * (a.wide ? 8 : 4);
        p.out = static_cast<char*>(a.out) + at * a.ldo * (a.out_bf16 ? 2 : 4);
        const dim3 grid(static_cast<uint32_t>(ceil_div(p.n, cut.rows(kThreads)) * cut.pieces));
        const auto kernel = a.wide ? (a.e_bf16 ? (a.out_bf16 ? embed_kernel<true, true, true> : embed_kernel<true, true, false>)
                                               : (a.out_bf16 ? embed_kernel<true, false, true> : embed_kernel<true, false, false>))
                                   : (a.e_bf16 ? (a.out_bf16 ? embed_kernel<false, true, true> : embed_kernel<false, true, false>)
                                               : (a.out_bf16 ? embed_kernel<false, false, true> : embed_kernel<false, false, false>));
        kernel<<<grid, kThreads, 0, st>>>(p, cut);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t embed_workspace_bytes(int64_t n, int64_t vocab, int64_t d) { return n == 0 || d == 0 ? 0 : plan_of(n, vocab, d).bytes(); }

bool embed_grad_fits(int64_t n, int64_t vocab, int64_t d) {
    const Plan p = plan_of(n, vocab, d);
    return grid_fits(ceil_div(vocab, fill_rows(vocab)) + sum_blocks(p), kThreads) && grid_fits(join_blocks(p, d), kThreads);
}

hipError_t launch_embed_grad(const EmbedGradArgs& a, hipStream_t st) {
    const Plan p = plan_of(a.n, a.vocab, a.d);
    uint32_t *keys = nullptr, *index = nullptr;
    if (a.n > 0) {
        const hipError_t e = a.wide ? sort_tokens<true>(a, p, keys, index, st) : sort_tokens<false>(a, p, keys, index, st);
        if (e != hipSuccess) return e;
    }
    if (a.g_bf16) return a.e_bf16 ? sum_rows<true, true>(a, p, keys, index, st) : sum_rows<true, false>(a, p, keys, index, st);
    return a.e_bf16 ? sum_rows<false, true>(a, p, keys, index, st) : sum_rows<false, false>(a, p, keys, index, st);
}

}  // namespace coded
