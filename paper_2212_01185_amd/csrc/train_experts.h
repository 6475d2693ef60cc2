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
// 64 entries at a time: equal experts of a wave are found by ballots over the bits of their numbers.
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
        uint32_t b = 0, t = 0;
        if (a.segments > 1) {
            for (uint32_t s = 0; s < a.segments; ++s) {
                const uint32_t c = a.counts[(size_t)s * experts + e];
                b += s < blockIdx.x ? c : 0;
                t += c;
            }
        } else {
            for (int w = 0; w < kSortWaves; ++w) t += sort_shared[w * experts + e];
        }
        before[e] = b;
        total[e] = t;
    }
    __syncthreads();
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
    uint32_t chunks;        // eights of a row
};
constexpr int kExpertThreads = 256;

// A thread has eight neighbours of a token's row.
template <class T>
__global__ __launch_bounds__(kExpertThreads) void expert_rows_kernel(Experts a) {
    const uint64_t id = (uint64_t)blockIdx.x * kExpertThreads + threadIdx.x, token = id / a.chunks;
    if (token >= a.tokens) return;
    const int f = 8 * (int)(id - token * a.chunks);
    Eight<T> x;
    x.load(a.x, token * a.ldx + f, a.features - f);
    for (int j = 0; j < a.k; ++j) {
        const uint32_t at = (uint32_t)a.place[token * a.k + j];
        if (at < a.rows) x.store(a.y, at * a.ldy + f, a.features - f);
    }
}

template <class T, class Y>
__global__ __launch_bounds__(kExpertThreads) void expert_join_kernel(Experts a) {
    const uint64_t id = (uint64_t)blockIdx.x * kExpertThreads + threadIdx.x, token = id / a.chunks;
    if (token >= a.tokens) return;
    const int f = 8 * (int)(id - token * a.chunks);
    float sum[8] = {};
    for (int j = 0; j < a.k; ++j) {
        const uint32_t at = (uint32_t)a.place[token * a.k + j];
        if (at >= a.rows) continue;
        const float w = a.weight ? a.weight[token * a.k + j] : 1.0f;
        Eight<T> z;
        z.load(a.z, at * a.ldz + f, a.features - f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __builtin_fmaf(w, z.get(e), sum[e]);
    }
    Eight<Y> y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y.set(e, sum[e]);
    y.store(a.y, token * a.ldy + f, a.features - f);
}

// A wave has a token.
template <class T, class Y>
__global__ __launch_bounds__(kExpertThreads) void expert_join_grad_kernel(Experts a) {
    const uint64_t token = (uint64_t)blockIdx.x * (kExpertThreads / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (token >= a.tokens) return;
    for (int j = 0; j < a.k; ++j) {
        const uint32_t at = (uint32_t)a.place[token * a.k + j];
        const bool there = at < a.rows;
        const float w = a.weight ? a.weight[token * a.k + j] : 1.0f;
        float dot = 0.0f;
        if (there)
            for (int f = 8 * lane; f < a.features; f += 512) {
                Eight<Y> dy;
                dy.load(a.x, token * a.ldx + f, a.features - f);
                if (a.dweight) {
                    Eight<T> z;
                    z.load(a.z, at * a.ldz + f, a.features - f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(dy.get(e), z.get(e), dot);
                }
                if (a.y) {
                    Eight<T> dz;
#pragma unroll
                    for (int e = 0; e < 8; ++e) dz.set(e, w * dy.get(e));
                    dz.store(a.y, at * a.ldy + f, a.features - f);
                }
            }
        if (a.dweight) {
            dot = lanes_sum<64>(dot);
            if (lane == 0) a.dweight[token * a.k + j] = there ? dot : 0.0f;
        }
    }
}

}  // namespace pcc_train
