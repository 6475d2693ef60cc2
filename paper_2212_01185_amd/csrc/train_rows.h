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

// (Values, not elements of a vector: __builtin_bit_cast takes the first one's place of such.)
__device__ __forceinline__ float as_float(uint32_t bits) { return __builtin_bit_cast(float, bits); }
__device__ __forceinline__ uint32_t as_bits(float v) { return __builtin_bit_cast(uint32_t, v); }

// 16 bytes at an address that an element of SIZE bytes may have.
template <int SIZE>
struct Anywhere;
template <>
struct Anywhere<2> {
    typedef u32x4 type __attribute__((aligned(2)));
};
template <>
struct Anywhere<4> {
    typedef u32x4 type __attribute__((aligned(4)));
};

// Eight values of a row as memory has them: 16 or 32 bytes, at any address that an element may have.
template <class T>
struct Eight {
    static constexpr int kWords = kIs32<T> ? 2 : 1;
    using Place = Anywhere<sizeof(element_of<T>)>;
    u32x4 words[kWords];

    __device__ __forceinline__ void load8(const element_of<T>* from) {
#pragma unroll
        for (int k = 0; k < kWords; ++k) words[k] = reinterpret_cast<const typename Place::type*>(from)[k];
    }
    __device__ __forceinline__ void store8(element_of<T>* to) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) reinterpret_cast<typename Place::type*>(to)[k] = words[k];
    }
    // Past the caches.
    __device__ __forceinline__ void store8_past(element_of<T>* to) const {
#pragma unroll
        for (int k = 0; k < kWords; ++k) __builtin_nontemporal_store(words[k], reinterpret_cast<typename Place::type*>(to) + k);
    }
    __device__ __forceinline__ element_of<T> element(int e) const {
        if constexpr (kIs32<T>) return as_float(words[e / 4][e % 4]);
        else return (u16)(words[0][e / 2] >> (16 * (e % 2)));
    }
    __device__ __forceinline__ void one(element_of<T> v) {      // the first, and zeros
        clear();
        if constexpr (kIs32<T>) words[0][0] = as_bits(v);
        else words[0][0] = v;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < kWords; ++k) words[k] = u32x4{0, 0, 0, 0};
    }
    // The n values from the element `at` on (8 at most), and zeros.
    __device__ __forceinline__ void load(const void* base, size_t at, int n) {
        const element_of<T>* from = static_cast<const element_of<T>*>(base) + at;
        if (n >= 8) {
            load8(from);
        } else {
            clear();
#pragma unroll
            for (int e = 0; e < 7; ++e) {
                if (e >= n) continue;
                if constexpr (kIs32<T>) words[e / 4][e % 4] = as_bits(from[e]);
                else words[0][e / 2] |= (uint32_t)from[e] << (16 * (e % 2));
            }
        }
    }
    __device__ __forceinline__ void store(void* base, size_t at, int n) const {
        element_of<T>* to = static_cast<element_of<T>*>(base) + at;
        if (n >= 8) {
            store8(to);
        } else {
#pragma unroll
            for (int e = 0; e < 7; ++e)
                if (e < n) to[e] = element(e);
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (kIs32<T>) return as_float(words[e / 4][e % 4]);
        else if constexpr (std::is_same_v<T, Bf16>) return as_float(e % 2 ? words[0][e / 2] & 0xFFFF0000u : words[0][e / 2] << 16);
        else return from16<T>((u16)(words[0][e / 2] >> (16 * (e % 2))));
    }
    // All eight, to the nearest, ties to even.
    __device__ __forceinline__ void set(const float (&v)[8]) {
        if constexpr (kIs32<T>) {
#pragma unroll
            for (int e = 0; e < 8; ++e) words[e / 4][e % 4] = as_bits(v[e]);
        } else {
            typedef __attribute__((ext_vector_type(2))) typename T::value pair;
#pragma unroll
            for (int e = 0; e < 8; e += 2) words[0][e / 2] = __builtin_bit_cast(uint32_t, pair{(typename T::value)v[e], (typename T::value)v[e + 1]});
        }
    }
};

// Sums over groups of G neighbouring lanes (a power of two), the same in each of them: lanes exchange within quads, halves of a row of
// 16 and rows by the vector ALU's own permutations, whole rows by swaps.  All lanes of a group have to be active.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true);
}
constexpr int kSwapPairs = 0xB1, kSwapTwos = 0x4E, kMirrorEight = 0x141, kMirrorRow = 0x140, kTurnEight = 0x128;

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
    static_assert(G >= 8, "a row has eight lanes at least");
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

// A row that LANES lanes (8 at least) share: lane l has the eights l, l + LANES, ..., N of them at most, and of the up to seven features behind the last
// whole eight the l-th.
struct Extent {
    int eights, rest;       // of a row; 0 for a row that is not there

    __device__ __forceinline__ Extent(int features, bool there) : eights(there ? features >> 3 : 0), rest(there ? features & 7 : 0) {}
    // Of a part of a row: `most` eights from eight c0 on, and in the last part the rest.
    __device__ __forceinline__ Extent(int features, int c0, int most, bool there) {
        const int left = (features >> 3) - c0;
        eights = !there ? 0 : left < most ? left : most;
        rest = there && left <= most ? features & 7 : 0;
    }
};

template <class T, int LANES, int N>
struct Row {
    static_assert(LANES >= 8, "the features behind the last eight have a lane each");
    Eight<T> v[N], tail;    // of the tail the first value

    // f(8, i) for the eights that are this lane's, then f(1, N) for its value of the rest; both numbers are types.
    template <int I = 0, class F>
    static __device__ __forceinline__ void each(int lane, Extent w, F&& f) {
        if constexpr (I < N) {
            if (lane + LANES * I < w.eights) f(std::integral_constant<int, 8>{}, std::integral_constant<int, I>{});
            each<I + 1>(lane, w, f);
        } else {
            if (lane < w.rest) f(std::integral_constant<int, 1>{}, std::integral_constant<int, N>{});
        }
    }
    template <int I>
    __device__ __forceinline__ Eight<T>& at(std::integral_constant<int, I>) {
        if constexpr (I < N) return v[I];
        else return tail;
    }
    __device__ __forceinline__ void load(const void* base, size_t at0, int lane, Extent w) {
        const element_of<T>* from = static_cast<const element_of<T>*>(base) + at0;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane + LANES * i < w.eights) v[i].load8(from + 8 * (lane + LANES * i));
        if (lane < w.rest) tail.one(from[8 * w.eights + lane]);
    }
    template <int I>
    __device__ __forceinline__ void store(std::integral_constant<int, I>, void* base, size_t at0, int lane, Extent w) const {
        element_of<T>* to = static_cast<element_of<T>*>(base) + at0;
        if constexpr (I < N) v[I].store8(to + 8 * (lane + LANES * I));
        else to[8 * w.eights + lane] = tail.element(0);
    }
    template <int I>
    __device__ __forceinline__ void store_past(std::integral_constant<int, I> i, void* base, size_t at0, int lane, Extent w) const {
        if constexpr (I < N) v[I].store8_past(static_cast<element_of<T>*>(base) + at0 + 8 * (lane + LANES * I));
        else store(i, base, at0, lane, w);
    }
    // What was made of the values is made anew behind this, not kept: a value takes half a register as it came.
    __device__ __forceinline__ void forget() {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < Eight<T>::kWords; ++k) asm("" : "+v"(v[i].words[k]));
    }
};

// Sums in fp32 of a row's features, as `Row` deals them out.
template <int LANES, int N>
struct Sums {
    float v[N][8], tail[8];

    template <int I>
    __device__ __forceinline__ float (&at(std::integral_constant<int, I>))[8] {
        if constexpr (I < N) return v[I];
        else return tail;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i][e] = 0.0f;
            tail[e] = 0.0f;
        }
    }
    // Over the rows of a wave.
    __device__ __forceinline__ void sum_groups() {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = groups_sum<LANES>(v[i][e]);
        tail[0] = groups_sum<LANES>(tail[0]);
    }
};

}  // namespace pcc_train
