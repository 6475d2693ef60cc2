// The choice of a few experts for each token, and its gradient.
//
// The k largest logits of a token are found one after the other; equal ones lowest index first.  A logit of -inf is never chosen, a NaN is
// above all numbers (so it shows in the weights).  With top the largest and e_i = exp(l_i - top), the weight of a chosen one is e_i over the sum of
// the chosen, or of all, e.
//   d l_i = w_i (dw_i - sum w dw) over the chosen, and with the softmax over all  d l_i = p_i ([i chosen] dw_i - sum w dw)
#pragma once

#include "train_rows.h"

namespace pcc_train {

struct Route {
    const void* logits;
    const float* dweight;
    int32_t* expert;
    float* weight;
    void* dlogits;
    size_t ldl, lddl;
    uint64_t tokens;
    int experts, k, over_all;
};
constexpr int kRouteThreads = 256;

// Bits that are ordered as the numbers are, a NaN last.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return v != v ? 0xFFFFFFFFu : b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t key) { return __builtin_bit_cast(float, key >> 31 ? key & 0x7FFFFFFFu : ~key); }
constexpr uint32_t kNever = 0x007FFFFFu;        // ordered(-inf)

// e^v for v <= 0 (and NaN), with what the rounding of v log2(e) left out.
__device__ __forceinline__ float exp_below(float v) {
    constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
    const float b = v < -120.0f ? -120.0f : v, t = b * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, __builtin_fmaf(b, 1.925962989e-8f, __builtin_fmaf(b, kLog2e, -t)) * kLn2, e);
}

// LANES lanes have a token, eight neighbouring logits each, N times.
template <class T, int LANES, int N>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(Route a) {
    const uint64_t t0 = (uint64_t)blockIdx.x * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const bool mine = t0 < a.tokens;
    const uint64_t t = mine ? t0 : a.tokens - 1;
    const int lane = threadIdx.x % LANES;
    uint32_t key[8 * N];
    float all = 0.0f, top = 0.0f, total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = 8 * (lane + LANES * i);
        Eight<T> l;
        l.load(a.logits, t * a.ldl + f, a.experts - f);
#pragma unroll
        for (int e = 0; e < 8; ++e) key[8 * i + e] = f + e < a.experts ? ordered(l.get(e)) : 0u;
    }
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < 8 * N; ++i) best = key[i] > best ? key[i] : best;
        best = over_lanes<LANES>(best, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
        uint32_t index = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 8 * N - 1; i >= 0; --i) index = key[i] == best ? (uint32_t)(8 * (lane + LANES * (i / 8)) + i % 8) : index;
        index = over_lanes<LANES>(index, [](uint32_t p, uint32_t q) { return p < q ? p : q; });
        const bool taken = best > kNever;
        if (j == 0) {
            top = taken ? unordered(best) : 0.0f;
            if (a.over_all) {
#pragma unroll
                for (int i = 0; i < 8 * N; ++i) all += key[i] > kNever ? exp_below(unordered(key[i]) - top) : 0.0f;
                all = lanes_sum<LANES>(all);
            }
        }
        const float size = taken ? exp_below(unordered(best) - top) : 0.0f;
        total += size;
        if (mine && lane == 0) {
            a.expert[t * a.k + j] = taken ? (int32_t)index : -1;
            a.weight[t * a.k + j] = size;
        }
#pragma unroll
        for (int i = 0; i < 8 * N; ++i)
            if ((uint32_t)(8 * (lane + LANES * (i / 8)) + i % 8) == index) key[i] = 0;
    }
    if (mine && lane == 0) {
        const float by = a.over_all ? all : total;
        for (int j = 0; j < a.k; ++j) {
            const float size = a.weight[t * a.k + j];
            a.weight[t * a.k + j] = a.expert[t * a.k + j] >= 0 ? size / by : 0.0f;
        }
    }
}

template <class T, int LANES, int N>
__global__ __launch_bounds__(kRouteThreads) void route_grad_kernel(Route a) {
    const uint64_t t0 = (uint64_t)blockIdx.x * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const bool mine = t0 < a.tokens;
    const uint64_t t = mine ? t0 : a.tokens - 1;
    const int lane = threadIdx.x % LANES;
    float p[8 * N], along = 0.0f;
    if (a.over_all) {
        uint32_t best = 0;
        float all = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            Eight<T> l;
            l.load(a.logits, t * a.ldl + f, a.experts - f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[8 * i + e] = f + e < a.experts ? l.get(e) : -__builtin_inff();
                const uint32_t o = ordered(p[8 * i + e]);
                best = o > best ? o : best;
            }
        }
        best = over_lanes<LANES>(best, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
        const float top = best > kNever ? unordered(best) : 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * N; ++i) {
            p[i] = p[i] == -__builtin_inff() ? 0.0f : exp_below(p[i] - top);
            all += p[i];
        }
        all = lanes_sum<LANES>(all);
        const float inverse = all == 0.0f ? 0.0f : 1.0f / all;
#pragma unroll
        for (int i = 0; i < 8 * N; ++i) p[i] *= inverse;
    }
    for (int j = 0; j < a.k; ++j)
        if (a.expert[t * a.k + j] >= 0) along += a.weight[t * a.k + j] * a.dweight[t * a.k + j];
    float d[8 * N];
#pragma unroll
    for (int i = 0; i < 8 * N; ++i) d[i] = a.over_all ? -along * p[i] : 0.0f;
    for (int j = 0; j < a.k; ++j) {
        const int expert = a.expert[t * a.k + j];
        const float w = a.weight[t * a.k + j], dw = a.dweight[t * a.k + j];
#pragma unroll
        for (int i = 0; i < 8 * N; ++i)
            if (8 * (lane + LANES * (i / 8)) + i % 8 == expert) d[i] = a.over_all ? p[i] * (dw - along) : w * (dw - along);
    }
    if (!mine) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = 8 * (lane + LANES * i);
        if (f >= a.experts) continue;
        Eight<T> out;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = d[8 * i + e];
        out.set(v);
        out.store(a.dlogits, t * a.lddl + f, a.experts - f);
    }
}

}  // namespace pcc_train
