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

// A logit and its expert as one whole number: larger for larger logits, and for lower experts where they are equal.  A logit of 16 bits leaves the
// last ten bits of its fp32 form free, which take the expert; one of fp32 takes 32 more.  0 is less than any.
template <class T>
struct RouteKey {
    using type = std::conditional_t<kIs32<T>, uint64_t, uint32_t>;
    static constexpr uint32_t kLow = 0x3FF;
    static_assert(PCC_MAX_EXPERTS <= kLow + 1, "an expert's number has ten bits");
    // What is not above is -inf.
    static constexpr type kNever = kIs32<T> ? 0x007FFFFFFFFFFFFFull : 0x007FFFFFu;

    // Bits that are ordered as the numbers are: both zeros are one, a NaN is the last.
    static __device__ __forceinline__ type of(float v, uint32_t expert) {
        const uint32_t b = as_bits(v != v ? __builtin_nanf("") : v + 0.0f), o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
        if constexpr (kIs32<T>) return (type)o << 32 | ~expert;
        else return (o & ~kLow) | (kLow ^ expert);
    }
    static __device__ __forceinline__ float logit(type key) {
        uint32_t o;
        if constexpr (kIs32<T>) o = (uint32_t)(key >> 32);
        else o = key >> 31 ? key & ~kLow : key | kLow;
        return as_float(o >> 31 ? o ^ 0x80000000u : ~o);
    }
    static __device__ __forceinline__ int expert(type key) { return (int)(kIs32<T> ? ~(uint32_t)key : kLow ^ ((uint32_t)key & kLow)); }
};

template <int G>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
    return over_lanes<G>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int G>
__device__ __forceinline__ uint64_t lanes_max(uint64_t v) {
    auto step = [&](uint32_t low, uint32_t high) {
        const uint64_t other = (uint64_t)high << 32 | low;
        v = other > v ? other : v;
    };
    auto low = [&] { return (uint32_t)v; };
    auto high = [&] { return (uint32_t)(v >> 32); };
    if constexpr (G >= 2) step(moved<kSwapPairs>(low()), moved<kSwapPairs>(high()));
    if constexpr (G >= 4) step(moved<kSwapTwos>(low()), moved<kSwapTwos>(high()));
    if constexpr (G >= 8) step(moved<kMirrorEight>(low()), moved<kMirrorEight>(high()));
    if constexpr (G >= 16) step(moved<kMirrorRow>(low()), moved<kMirrorRow>(high()));
    if constexpr (G >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(low(), low(), false, false), q = __builtin_amdgcn_permlane16_swap(high(), high(), false, false);
        v = (uint64_t)q[0] << 32 | p[0];
        step(p[1], q[1]);
    }
    if constexpr (G >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(low(), low(), false, false), q = __builtin_amdgcn_permlane32_swap(high(), high(), false, false);
        v = (uint64_t)q[0] << 32 | p[0];
        step(p[1], q[1]);
    }
    return v;
}

// Eight keys, the largest first (merging by odd and even places, 19 comparisons).
template <class K>
__device__ __forceinline__ void sort_eight(K (&k)[8]) {
    constexpr int kPairs[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                   {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int i = 0; i < 19; ++i) {
        const K a = k[kPairs[i][0]], b = k[kPairs[i][1]];
        k[kPairs[i][0]] = a > b ? a : b;
        k[kPairs[i][1]] = a > b ? b : a;
    }
}

// e^v for v <= 0 (-inf gives 0), rounded as v log2(e) is: off by |v| half steps of fp32 beside its own.  A NaN stays one.
__device__ __forceinline__ float exp_below(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896341f); }

// Eight logits of a token from expert f on; what lies behind the last expert is -inf.
template <class T>
__device__ __forceinline__ void load_logits(Eight<T>& l, const Route& a, uint64_t t, int f, bool whole) {
    l.load(a.logits, t * a.ldl + f, a.experts - f);
    if (whole) return;
    constexpr uint32_t kBelow = kIs32<T> ? 0xFF800000u : std::is_same_v<T, Bf16> ? 0xFF80u : 0xFC00u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (kIs32<T>) l.words[e / 4][e % 4] = f + e < a.experts ? l.words[e / 4][e % 4] : kBelow;
        else l.words[0][e / 2] |= f + e < a.experts ? 0u : kBelow << (16 * (e % 2));     // (zeros until then)
    }
}

// Takes `best` off the lists that it is the first of; NEEDED entries of a list behind it are.
template <int NEEDED, class K, int N>
__device__ __forceinline__ void take_off(K (&key)[N][8], K best) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool taken = key[i][0] == best;
#pragma unroll
        for (int e = 0; e < (NEEDED < 8 ? NEEDED : 8); ++e) key[i][e] = taken ? (e < 7 ? key[i][e < 7 ? e + 1 : 7] : K{0}) : key[i][e];
    }
}
template <int LANES, class K, int N>
__device__ __forceinline__ K first_of(const K (&key)[N][8]) {
    K best = key[0][0];
#pragma unroll
    for (int i = 1; i < N; ++i) best = key[i][0] > best ? key[i][0] : best;
    return lanes_max<LANES>(best);
}
// Choices J, J + 1, ... of eight at most.
template <int LANES, int SLOTS, int J = 0, class K, int N>
__device__ __forceinline__ void choose_eight(K (&key)[N][8], K (&held)[SLOTS], K& top, int k, int lane) {
    if constexpr (J < 8) {
        if (J >= k) return;
        const K best = first_of<LANES>(key);
        if (J == 0) top = best;
        if (lane == J % LANES) held[J / LANES] = best;
        take_off<7 - J>(key, best);
        choose_eight<LANES, SLOTS, J + 1>(key, held, top, k, lane);
    }
}

// LANES lanes have a token, eight neighbouring logits each, N times.  Each lane sorts its own; then the largest of all lanes' first ones is taken off
// its list, k times, and choice j is kept by lane j % LANES.  Many tokens keep the vector ALU busy all the time: 393,216 tokens of 64 in bf16, 8 chosen, 24 us,
// 3.2 TB/s (searching all logits for each choice: 60), in fp32, whose keys take two registers, 33 us, 3.8 TB/s.
template <class T, int LANES, int N>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(Route a) {
    using Key = RouteKey<T>;
    using K = typename Key::type;
    constexpr int kSlots = LANES >= PCC_MAX_CHOICES ? 1 : LANES == 1 ? 8 : PCC_MAX_CHOICES / LANES;    // (k is at most the number of experts)
    const uint64_t t0 = (uint64_t)blockIdx.x * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const bool mine = t0 < a.tokens;
    const uint64_t t = mine ? t0 : a.tokens - 1;
    const int lane = threadIdx.x % LANES;
    const bool whole = a.experts == 8 * LANES * N;
    Eight<T> l[N];
    K key[N][8], held[kSlots] = {}, top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = 8 * (lane + LANES * i);
        load_logits(l[i], a, t, f, whole);
#pragma unroll
        for (int e = 0; e < 8; ++e) key[i][e] = Key::of(l[i].get(e), (uint32_t)(f + e));
        sort_eight(key[i]);
    }
    if (LANES == 1 || a.k <= 8) {
        choose_eight<LANES, kSlots>(key, held, top, a.k, lane);
    } else {
#pragma unroll
        for (int s = 0; s < kSlots; ++s)
            for (int u = 0; u < LANES && s * LANES + u < a.k; ++u) {
                const K best = first_of<LANES>(key);
                if (s == 0 && u == 0) top = best;
                if (lane == u) held[s] = best;
                take_off<8>(key, best);
            }
    }
    const bool some = top > Key::kNever;
    const float highest = some ? Key::logit(top) : 0.0f;
    float total = 0.0f, size[kSlots];
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        if (s * LANES >= a.k) break;
        size[s] = held[s] > Key::kNever ? exp_below(Key::logit(held[s]) - highest) : 0.0f;
        total += size[s];
    }
    if (a.over_all) {
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) total += exp_below(l[i].get(e) - highest);
    }
    const float inverse = 1.0f / lanes_sum<LANES>(total);      // (a weight is a product with it: two roundings where a quotient has one)
    if (!mine) return;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        if (s * LANES >= a.k) break;
        const int j = s * LANES + lane;
        if (j >= a.k) continue;
        a.expert[t * a.k + j] = held[s] > Key::kNever ? Key::expert(held[s]) : -1;
        a.weight[t * a.k + j] = held[s] > Key::kNever ? size[s] * inverse : 0.0f;
    }
}

// A wave's tokens have a place in LDS for each logit: zeros, then what each choice brings is put in its expert's, by the lane that kept it.  393,216 tokens of
// 64 in bf16, 8 chosen, softmax over all: 22 us, 6.2 TB/s with what the caches hold (each lane comparing its logits' numbers with every choice: 53).
template <class T, int LANES, int N>
__global__ __launch_bounds__(kRouteThreads) void route_grad_kernel(Route a) {
    constexpr int kSlots = LANES >= PCC_MAX_CHOICES ? 1 : LANES == 1 ? 8 : PCC_MAX_CHOICES / LANES;
    __shared__ __align__(16) float brought[kRouteThreads * 8 * N];
    const uint64_t t0 = (uint64_t)blockIdx.x * (kRouteThreads / LANES) + threadIdx.x / LANES;
    const bool mine = t0 < a.tokens;
    const uint64_t t = mine ? t0 : a.tokens - 1;
    const int lane = threadIdx.x % LANES;
    const bool whole = a.experts == 8 * LANES * N;
    float* own = brought + threadIdx.x / LANES * (LANES * 8 * N);
    Eight<T> l[N];
    int expert[kSlots];
    float w[kSlots], dw[kSlots], along = 0.0f;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        expert[s] = -1;
        if (s * LANES >= a.k) break;
        const int j = s * LANES + lane;
        const bool there = j < a.k;
        expert[s] = there ? a.expert[t * a.k + j] : -1;
        w[s] = there ? a.weight[t * a.k + j] : 0.0f;
        dw[s] = there ? a.dweight[t * a.k + j] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = 8 * (lane + LANES * i);
        if (a.over_all) load_logits(l[i], a, t, f, whole);
        f32x4* zeros = reinterpret_cast<f32x4*>(own + f);
        zeros[0] = zeros[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
        if (s * LANES >= a.k) break;
        if ((uint32_t)expert[s] >= (uint32_t)a.experts) expert[s] = -1;
        along += expert[s] >= 0 ? w[s] * dw[s] : 0.0f;
    }
    along = lanes_sum<LANES>(along);
    __builtin_amdgcn_wave_barrier();        // a token's lanes are in one wave
#pragma unroll
    for (int s = 0; s < kSlots; ++s)
        if (s * LANES < a.k && expert[s] >= 0) own[expert[s]] = a.over_all ? dw[s] : w[s] * (dw[s] - along);
    float top = -__builtin_inff(), all = 0.0f;
    if (a.over_all) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = l[i].get(e);
                top = v > top ? v : top;        // (a NaN does not become the largest: it shows in the sum)
            }
        top = over_lanes<LANES>(top, [](float x, float y) { return x > y ? x : y; });
        top = top == -__builtin_inff() ? 0.0f : top;
    }
    float p[N][8];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[i][e] = a.over_all ? exp_below(l[i].get(e) - top) : 0.0f;
            all += p[i][e];
        }
    all = lanes_sum<LANES>(all);
    const float inverse = all == 0.0f ? 0.0f : 1.0f / all;
    __builtin_amdgcn_wave_barrier();
    if (!mine) return;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int f = 8 * (lane + LANES * i);
        if (f >= a.experts) continue;
        const f32x4 low = *reinterpret_cast<const f32x4*>(own + f), high = *reinterpret_cast<const f32x4*>(own + f + 4);
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float g = e < 4 ? low[e] : high[e - 4];
            // (a masked logit's 0 is no product: along or the sum may be infinite or NaN)
            d[e] = !a.over_all ? g : l[i].get(e) == -__builtin_inff() ? 0.0f : p[i][e] * inverse * (g - along);
        }
        Eight<T> out;
        out.set(d);
        out.store(a.dlogits, t * a.lddl + f, a.experts - f);
    }
}

}  // namespace pcc_train
