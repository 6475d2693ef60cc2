// Tokens sorted by expert, laid out as rows, and the experts' rows joined by token.
//
// An entry is a token's j-th choice; place[entry] is its row: entries of lower experts first, those of one expert in their own order.  An entry that
// names no expert has place -1.
//   rows      rows[place] = x[token]
//   join      y[token] = sum over j of weight z[place]       (its gradient: dz[place] = weight dy[token], dweight = dy[token] . z[place])
#pragma once

#include "train_rows.h"

namespace pcc_train {

// ---------------------------------------------------------------------------
// Sort by counting.  A workgroup of 16 waves has a segment of the entries, a wave a sixteenth of it.  The first kernel counts each segment's
// experts; in the second a workgroup finds by those counts where its entries of each expert go, then its waves deal the places out
// 64 entries at a time: equal experts of a wave are found by ballots over the bits of their numbers.  One segment (4,096 entries) takes the second kernel alone.
// 786,432 entries of 16 experts: 5 and 7 us, of which the entries' bytes are one (a thread an expert for the sum over segments: 36 instead of 7).
// ---------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;

struct Sort {
    const int32_t* expert;
    int64_t* offsets;
    int32_t* place;
    uint32_t* counts;       // [segments][experts]
    uint32_t entries, segment;      // a segment: a multiple of 1024 entries
    uint32_t segments;
    int experts, bits;      // bits: of the experts' numbers and one more
};

__device__ __forceinline__ int expert_of(const Sort& a, uint32_t i, uint32_t end) {     // experts: none
    const int e = i < end ? a.expert[i] : -1;
    return (uint32_t)e < (uint32_t)a.experts ? e : a.experts;
}

__global__ __launch_bounds__(kSortThreads) void expert_count_kernel(Sort a) {
    extern __shared__ __align__(16) uint32_t sort_shared[];
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads) sort_shared[e] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.segment, end = a.entries - begin < a.segment ? a.entries : begin + a.segment;
    for (uint32_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const int e = expert_of(a, i, end);
        if (e < a.experts) atomicAdd(&sort_shared[e], 1u);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.experts; e += kSortThreads) a.counts[(size_t)blockIdx.x * a.experts + e] = sort_shared[e];
}

// LDS: places of each wave and expert, then two values an expert, then the sums of the waves.
__host__ __device__ constexpr size_t sort_lds(int experts) { return ((size_t)(kSortWaves + 2) * experts + kSortWaves) * sizeof(uint32_t); }

__global__ __launch_bounds__(kSortThreads) void expert_place_kernel(Sort a) {
    extern __shared__ __align__(16) uint32_t sort_shared[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, experts = a.experts;
    uint32_t* mine = sort_shared + wave * experts;
    uint32_t* before = sort_shared + kSortWaves * experts;      // entries of the expert in the segments in front
    uint32_t* total = before + experts;                         // in all of them; then those of lower experts
    uint32_t* sums = total + experts;
    for (int i = threadIdx.x; i < kSortWaves * experts; i += kSortThreads) sort_shared[i] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * a.segment, end = a.entries - begin < a.segment ? a.entries : begin + a.segment, part = a.segment / kSortWaves;
    const uint32_t from = begin + wave * part, to = from + part < end ? from + part : end;
    for (uint32_t i = from + lane; i < to; i += 64) {
        const int e = expert_of(a, i, to);
        if (e < experts) atomicAdd(&mine[e], 1u);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kSortThreads) {
        uint32_t t = 0;
        if (a.segments == 1)
            for (int w = 0; w < kSortWaves; ++w) t += sort_shared[w * experts + e];
        before[e] = 0;
        total[e] = t;
    }
    __syncthreads();
    if (a.segments > 1) {
        // a thread has an expert and every so many-th segment
        const int slices = kSortThreads / experts, e = threadIdx.x % experts, slice = threadIdx.x / experts;
        uint32_t b = 0, t = 0;
        if (slice < slices) {
#pragma unroll 8
            for (uint32_t s = slice; s < a.segments; s += slices) {
                const uint32_t c = a.counts[(size_t)s * experts + e];
                b += s < blockIdx.x ? c : 0;
                t += c;
            }
            atomicAdd(&before[e], b);       // whole numbers: in any order
            atomicAdd(&total[e], t);
        }
        __syncthreads();
    }
    // sums of the experts in front; there are at most as many as threads
    uint32_t own = (int)threadIdx.x < experts ? total[threadIdx.x] : 0, sum = wave_prefix(own);
    if (lane == 63) sums[wave] = sum;
    __syncthreads();
    uint32_t front = sum - own;
    for (int w = 0; w < wave; ++w) front += sums[w];
    if ((int)threadIdx.x < experts) {
        const int e = threadIdx.x;
        if (blockIdx.x == 0) {
            a.offsets[e] = front;
            if (e + 1 == experts) a.offsets[experts] = front + own;
        }
        uint32_t at = front + before[e];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = sort_shared[w * experts + e];
            sort_shared[w * experts + e] = at;
            at += c;
        }
    }
    __syncthreads();
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const uint32_t i = i0 + lane;
        const int e = expert_of(a, i, to);
        uint64_t same = ~0ull;
        for (int b = 0; b < a.bits; ++b) {
            const bool bit = (e >> b) & 1;
            const uint64_t set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        uint32_t at = 0;
        if (e < experts) at = mine[e];
        __builtin_amdgcn_wave_barrier();
        if (e < experts && rank == 0) mine[e] = at + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (i < to) a.place[i] = e < experts ? (int32_t)(at + rank) : -1;
    }
}

// ---------------------------------------------------------------------------
// Rows.
// ---------------------------------------------------------------------------
struct Experts {
    const void* x;          // tokens: x, dy
    const void* z;          // rows
    const int32_t* place;
    const float* weight;    // or null: 1
    void* y;                // rows: the rows; join: y; its gradient: dz, or null
    float* dweight;         // or null
    size_t ldx, ldz, ldy;
    uint64_t tokens, rows;
    int k, features;
    uint32_t each;          // workgroups for each of the chip's eight dies
};
constexpr int kExpertThreads = 256;

// Memory bounds all of these.  us, 393,216 tokens with 2 rows of 160 in bf16 each: rows 69 (5.4 TB/s), join 72 (5.3), its gradient 124 (5.1); 8,192 tokens with
// four of 2,048, join to fp32, 43 (4.6).
// A token's row has LANES lanes, parts of LANES * N eights one after the other.  A die has neighbouring tokens, whose rows of one expert are neighbours
// as well and share lines of its L2.
template <int LANES>
__device__ __forceinline__ uint64_t token_of(const Experts& a) {
    constexpr int kTeams = kExpertThreads / LANES;
    return ((uint64_t)(blockIdx.x % 8) * a.each + blockIdx.x / 8) * kTeams + threadIdx.x / LANES;
}

template <class T, int LANES, int N, bool PAST>
__global__ __launch_bounds__(kExpertThreads) void expert_rows_kernel(Experts a) {
    const uint64_t token = token_of<LANES>(a);
    if (token >= a.tokens) return;
    const int lane = threadIdx.x % LANES;
    const int32_t* place = a.place + token * a.k;
    for (int c0 = 0; c0 == 0 || c0 < a.features >> 3; c0 += LANES * N) {
        const Extent w(a.features, c0, LANES * N, true);
        Row<T, LANES, N> x;
        x.load(a.x, token * a.ldx + 8 * c0, lane, w);
        for (int j = 0; j < a.k; ++j) {
            const uint32_t at = (uint32_t)place[j];
            if (at < a.rows)
                Row<T, LANES, N>::each(lane, w, [&](auto, auto i) {
                    if constexpr (PAST) x.store_past(i, a.y, at * a.ldy + 8 * c0, lane, w);
                    else x.store(i, a.y, at * a.ldy + 8 * c0, lane, w);
                });
        }
    }
}

template <class T, class Y, int LANES, int N>
__global__ __launch_bounds__(kExpertThreads) void expert_join_kernel(Experts a) {
    constexpr int kAtOnce = N == 1 ? 4 : 2;         // rows on their way
    using Z = Row<T, LANES, N>;
    const uint64_t token = token_of<LANES>(a);
    if (token >= a.tokens) return;
    const int lane = threadIdx.x % LANES;
    for (int c0 = 0; c0 == 0 || c0 < a.features >> 3; c0 += LANES * N) {
        const Extent w(a.features, c0, LANES * N, true);
        Sums<LANES, N> sum;
        sum.clear();
        for (int j0 = 0; j0 < a.k; j0 += kAtOnce) {
            Z z[kAtOnce];
            float weight[kAtOnce];
            bool there[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const bool more = j0 + j < a.k;
                const uint32_t at = more ? (uint32_t)a.place[token * a.k + j0 + j] : ~0u;
                there[j] = at < a.rows;
                weight[j] = more && a.weight ? a.weight[token * a.k + j0 + j] : 1.0f;
                z[j].load(a.z, at * a.ldz + 8 * c0, lane, Extent(a.features, c0, LANES * N, there[j]));
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                Z::each(lane, Extent(a.features, c0, LANES * N, there[j]), [&](auto wide, auto i) {
#pragma unroll
                    for (int e = 0; e < wide; ++e) sum.at(i)[e] = __builtin_fmaf(weight[j], z[j].at(i).get(e), sum.at(i)[e]);
                });
        }
        Row<Y, LANES, N> y;
        Z::each(lane, w, [&](auto, auto i) {
            y.at(i).set(sum.at(i));
            // past the caches, us so and not: 393,216 rows of 160 in bf16 72 and 76, 8,192 of 2,048 in fp32 43 and 46 (but 44 and 40 where three sets of
            // inputs and results are all there is, and the last results still lie in the caches when they are written again).  With dropout and its residual
            // behind it, in a graph: 300 of 160 in bf16 4.9 and 4.7, 393,216 of 160 141 and 137, 1,024 of 2,048 in fp32 12.9 and 13.9, 8,192 of them 74 and 74
            y.store_past(i, a.y, token * a.ldy + 8 * c0, lane, w);
        });
    }
}

template <class T, class Y, int LANES, int N>
__global__ __launch_bounds__(kExpertThreads) void expert_join_grad_kernel(Experts a) {
    constexpr int kAtOnce = N == 1 ? 4 : 2, kWaves = LANES <= 64 ? 1 : LANES / 64;
    using Z = Row<T, LANES, N>;
    __shared__ float meet[2][kAtOnce][kWaves];
    const uint64_t token = token_of<LANES>(a);
    const bool mine = token < a.tokens;
    const int lane = threadIdx.x % LANES, k = mine ? a.k : 0, most = LANES * N;
    const bool one = (a.features >> 3) <= most;         // the whole row at once: dy is read once
    Row<Y, LANES, N> dy;
    if (one) dy.load(a.x, token * a.ldx, lane, Extent(a.features, mine));
    int turn = 0;
    for (int j0 = 0; j0 < a.k; j0 += kAtOnce, turn ^= 1) {
        uint32_t at[kAtOnce];
        float weight[kAtOnce], dot[kAtOnce] = {};
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            at[j] = j0 + j < k ? (uint32_t)a.place[token * a.k + j0 + j] : ~0u;
            weight[j] = j0 + j < k && a.weight ? a.weight[token * a.k + j0 + j] : 1.0f;
        }
        for (int c0 = 0; c0 == 0 || c0 < a.features >> 3; c0 += most) {
            if (!one) dy.load(a.x, token * a.ldx + 8 * c0, lane, Extent(a.features, c0, most, mine));
            Z z[kAtOnce];
            if (a.dweight)
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) z[j].load(a.z, at[j] * a.ldz + 8 * c0, lane, Extent(a.features, c0, most, at[j] < a.rows));
            if (a.y)
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const Extent w(a.features, c0, most, at[j] < a.rows);
                    Z dz;
                    Z::each(lane, w, [&](auto wide, auto i) {
                        float v[8] = {};
#pragma unroll
                        for (int e = 0; e < wide; ++e) v[e] = weight[j] * dy.at(i).get(e);
                        dz.at(i).set(v);
                        dz.store(i, a.y, at[j] * a.ldy + 8 * c0, lane, w);
                    });
                }
            if (a.dweight)
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    Z::each(lane, Extent(a.features, c0, most, at[j] < a.rows), [&](auto wide, auto i) {
#pragma unroll
                        for (int e = 0; e < wide; ++e) dot[j] = __builtin_fmaf(dy.at(i).get(e), z[j].at(i).get(e), dot[j]);
                    });
        }
        if (!a.dweight) continue;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            dot[j] = lanes_sum<(LANES < 64 ? LANES : 64)>(dot[j]);
            if (kWaves > 1 && (threadIdx.x & 63) == 0) meet[turn][j][lane >> 6] = dot[j];
        }
        if constexpr (kWaves > 1) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                dot[j] = 0.0f;
#pragma unroll
                for (int v = 0; v < kWaves; ++v) dot[j] += meet[turn][j][v];
            }
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (lane == j && j0 + j < k) a.dweight[token * a.k + j0 + j] = dot[j];
    }
}

}  // namespace pcc_train
