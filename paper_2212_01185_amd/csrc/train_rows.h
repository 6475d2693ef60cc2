// What the kernels that work along rows share: eight neighbouring values at a time, at any address, and sums over the lanes that
// have a row.
#pragma once

#include <type_traits>

#include "train_device.h"

namespace pcc_train {

struct Fp32 {
    typedef float value;
};

template <class T>
constexpr bool kIs32 = std::is_same_v<T, Fp32>;
template <class T>
using element_of = std::conditional_t<kIs32<T>, float, u16>;

// Eight values of a row as memory has them: 16 or 32 bytes.
template <class T>
struct Eight {
    element_of<T> v[8];

    // From the element `at` on, n of them (8 at most), and zeros.  Whole ones are one load (two of fp32) at any address.
    __device__ __forceinline__ void load(const void* base, size_t at, int n) {
        const element_of<T>* from = static_cast<const element_of<T>*>(base) + at;
        if (n >= 8) {
            __builtin_memcpy(v, from, sizeof(v));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? from[e] : element_of<T>{};
        }
    }
    __device__ __forceinline__ void store(void* base, size_t at, int n) const {
        element_of<T>* to = static_cast<element_of<T>*>(base) + at;
        if (n >= 8) {
            __builtin_memcpy(to, v, sizeof(v));
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < n) to[e] = v[e];
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (kIs32<T>) return v[e];
        else return from16<T>(v[e]);
    }
    __device__ __forceinline__ void set(int e, float value) {       // to the nearest, ties to even
        if constexpr (kIs32<T>) v[e] = value;
        else v[e] = to16<T>(value);
    }
};

// A row that LANES lanes (8 at least) share: lane l has the eights l, l + LANES, ..., N of them at most, and of the up to seven features behind the last
// whole eight the l-th.
struct Extent {
    int eights, rest;       // of a row; 0 for a row that is not there

    __device__ __forceinline__ Extent(int features, bool there) : eights(there ? features >> 3 : 0), rest(there ? features & 7 : 0) {}
};

template <class T, int LANES, int N>
struct Row {
    static_assert(LANES >= 8, "the features behind the last eight have a lane each");
    Eight<T> v[N];
    Eight<T> tail;          // the first value

    // f(i, eight) for the eights that are this lane's, then f(N, eight of one value) for its value of the rest.
    template <class F>
    static __device__ __forceinline__ void each(int lane, Extent w, F&& f) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane + LANES * i < w.eights) f(std::integral_constant<int, 8>{}, i);
        if (lane < w.rest) f(std::integral_constant<int, 1>{}, N);
    }
    __device__ __forceinline__ Eight<T>& at(int i) { return i < N ? v[i < N ? i : 0] : tail; }
    __device__ __forceinline__ const Eight<T>& at(int i) const { return i < N ? v[i < N ? i : 0] : tail; }

    __device__ __forceinline__ void load(const void* base, size_t at0, int lane, Extent w) {
        const element_of<T>* from = static_cast<const element_of<T>*>(base) + at0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane + LANES * i < w.eights) __builtin_memcpy(v[i].v, from + 8 * (lane + LANES * i), sizeof(v[i].v));
        if (lane < w.rest) tail.v[0] = from[8 * w.eights + lane];
    }
    __device__ __forceinline__ void store(int i, void* base, size_t at0, int lane, Extent w) const {
        element_of<T>* to = static_cast<element_of<T>*>(base) + at0;
        if (i < N) __builtin_memcpy(to + 8 * (lane + LANES * i), v[i < N ? i : 0].v, sizeof(v[0].v));
        else to[8 * w.eights + lane] = tail.v[0];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i].v[e] = element_of<T>{};
        tail.v[0] = element_of<T>{};
    }
    // What was made of the values is made anew behind this, not kept: a value takes half a register as it came.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            constexpr int kWords = sizeof(v[0].v) / 16;
            u32x4 words[kWords];
            __builtin_memcpy(words, v[i].v, sizeof(words));
#pragma unroll
            for (int k = 0; k < kWords; ++k) asm("" : "+v"(words[k]));
            __builtin_memcpy(v[i].v, words, sizeof(words));
        }
    }
};

// Sums over groups of G neighbouring lanes (a power of two), the same in each of them: lanes exchange within quads, halves of a row of
// 16 and rows by the vector ALU's own permutations, whole rows by swaps.  All lanes of a group have to be active.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
constexpr int kSwapPairs = 0xB1, kSwapTwos = 0x4E, kMirrorEight = 0x141, kMirrorRow = 0x140, kTurnFour = 0x124, kTurnEight = 0x128;

template <int G, class V, class F>
__device__ __forceinline__ V over_lanes(V v, F&& join) {
    static_assert(sizeof(V) == 4, "lanes exchange 32 bits");
    auto bits = [](V x) { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) { return __builtin_bit_cast(V, x); };
    if constexpr (G >= 2) v = join(v, value(moved<kSwapPairs>(bits(v))));
    if constexpr (G >= 4) v = join(v, value(moved<kSwapTwos>(bits(v))));
    if constexpr (G >= 8) v = join(v, value(moved<kMirrorEight>(bits(v))));
    if constexpr (G >= 16) v = join(v, value(moved<kMirrorRow>(bits(v))));
    if constexpr (G >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        v = join(value(p[0]), value(p[1]));
    }
    if constexpr (G >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        v = join(value(p[0]), value(p[1]));
    }
    return v;
}
template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
    return over_lanes<G>(v, [](float a, float b) { return a + b; });
}
// Sums over the lanes of a wave that have the same place in their group of G.
template <int G>
__device__ __forceinline__ float groups_sum(float v) {
    auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
    auto value = [](uint32_t x) { return __builtin_bit_cast(float, x); };
    if constexpr (G <= 4) v += value(moved<kTurnFour>(bits(v)));
    if constexpr (G <= 8) v += value(moved<kTurnEight>(bits(v)));
    if constexpr (G <= 16) {
        const auto p = __builtin_amdgcn_permlane16_swap(bits(v), bits(v), false, false);
        v = value(p[0]) + value(p[1]);
    }
    if constexpr (G <= 32) {
        const auto p = __builtin_amdgcn_permlane32_swap(bits(v), bits(v), false, false);
        v = value(p[0]) + value(p[1]);
    }
    return v;
}

}  // namespace pcc_train
