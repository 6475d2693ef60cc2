// What the kernels of a training step share: 16-bit types, the activations, the order of ragged groups of rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pcc.h"

namespace pcc_train {

// ---------------------------------------------------------------------------
// 16-bit types.  A value is carried as its bits (u16); F<T> names the arithmetic.
// ---------------------------------------------------------------------------
typedef uint16_t u16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) u16 u16x4;
typedef __attribute__((ext_vector_type(8))) u16 u16x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Bf16 {
    typedef __bf16 value;
    typedef __attribute__((ext_vector_type(8))) __bf16 operand;
    __device__ static f32x4 mfma(u16x8 a, u16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(operand, a), __builtin_bit_cast(operand, b), c, 0, 0, 0);
    }
    static constexpr u16 kOne = 0x3F80;
};
struct Fp16 {
    typedef _Float16 value;
    typedef __attribute__((ext_vector_type(8))) _Float16 operand;
    __device__ static f32x4 mfma(u16x8 a, u16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(operand, a), __builtin_bit_cast(operand, b), c, 0, 0, 0);
    }
    static constexpr u16 kOne = 0x3C00;
};

// To 16 bits, to the nearest, ties to even: what the products' operands are made of.
template <class T>
__device__ __forceinline__ u16 to16(float v) {
    return __builtin_bit_cast(u16, (typename T::value)v);
}
template <class T>
__device__ __forceinline__ float from16(u16 v) {
    return (float)__builtin_bit_cast(typename T::value, v);
}

// ReLU and LeakyReLU (slope 0.01) as the codec's network has them; a NaN stays one.
constexpr float kLeakySlope = 0.01f;
__device__ __forceinline__ float activate(float z, int act) {
    if (act == PCC_ACT_NONE) return z;
    return z < 0.0f ? (act == PCC_ACT_RELU ? 0.0f : kLeakySlope * z) : z;
}
// Times the derivative of the activation whose result is x.  Both activations keep the sign, so x tells; at 0 it is that
// of the negative side.
__device__ __forceinline__ float times_derivative(float d, float x, int act) {
    return act == PCC_ACT_NONE || x > 0.0f ? d : act == PCC_ACT_RELU ? 0.0f : kLeakySlope * d;
}

// ---------------------------------------------------------------------------
// Ragged groups.  off[0..groups] are device data, so no launch knows the groups' sizes: a launch has a workgroup for
// every chunk of mult * 2^log2 rows that could exist (rows / that, and one more a group for the parts), and a
// workgroup looks up which rows are its own.  Offsets are clamped to the rows there are and to rising order, so
// that wrong ones make wrong results but no access outside the tensors.
// ---------------------------------------------------------------------------
struct Chunk {
    int group;          // -1: there is no such chunk
    int64_t lo, hi;     // rows
    uint32_t shared;    // number of the chunk among those of groups that have more than one
    uint32_t count;     // chunks of the group
    uint32_t part;      // tile of the chunk
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    return (int64_t)(((uint64_t)uniform((uint32_t)((uint64_t)v >> 32)) << 32) | uniform((uint32_t)(uint64_t)v));
}

// Rows of group g and how many chunks they make; with `empty`, a group without rows has one, of no rows.
__device__ __forceinline__ uint32_t group_chunks(const int64_t* __restrict__ off, int g, int groups, int64_t rows, int log2, uint32_t mult, bool empty, int64_t& lo, int64_t& hi) {
    if (g >= groups) { lo = hi = 0; return 0; }
    lo = clamp64(off[g], 0, rows);
    hi = clamp64(off[g + 1], lo, rows);
    const uint32_t n = ((uint32_t)((hi - lo + ((int64_t)1 << log2) - 1) >> log2) + mult - 1) / mult;
    return empty && n == 0 ? 1 : n;
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += (uint32_t)__shfl_xor((int)v, d);
    return uniform(v);
}
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = (uint32_t)__shfl_up((int)v, d);
        if (lane >= d) v += up;
    }
    return v;
}

// Where a group's chunks begin in an order that its offset alone tells: group g has the places from `place`(g) to `place`(g + 1), one more than it
// needs at most, since a row at the offset a of chunks of c rows has a / c chunks in front of it and each group adds one for its part.
__device__ __forceinline__ uint32_t whole_chunks(int64_t rows, int log2, uint32_t mult) { return (uint32_t)(rows >> log2) / mult; }
__device__ __forceinline__ uint32_t place(const int64_t* __restrict__ off, int g, int64_t rows, int log2, uint32_t mult) {
    return whole_chunks(clamp64(off[g], 0, rows), log2, mult) + (uint32_t)g;
}
// The same for the sums of groups of more than one chunk, where there are more than 64 groups: within the workspace's rows / c + groups, or 2 rows / c
// (such a group of n chunks has an offset c behind its own at least, and n <= 2 (b / c - a / c)).
__device__ __forceinline__ uint32_t shared_place(int64_t lo, int g, int groups, int64_t rows, int log2, uint32_t mult) {
    const uint32_t before = whole_chunks(lo, log2, mult);
    return (uint32_t)groups <= whole_chunks(rows, log2, mult) ? before + (uint32_t)g : 2 * before;
}

// find_chunk for more than 64 groups: searched 64 at a time by their places (65,535 in three steps), some of which hold no chunk.  Numbering the
// chunks as they are would take every workgroup through all offsets (65,535 rows of 32 to 32, us, numbered and so: 4,096 groups 540 and 32, 65,535
// groups 131,000 and 445).
__device__ __forceinline__ Chunk search_chunk(const int64_t* __restrict__ off, int groups, int64_t rows, int log2, uint32_t mult, uint32_t tiles, uint32_t b, bool empty) {
    const Chunk none = {-1, 0, 0, 0, 0, 0};
    const int lane = threadIdx.x & 63;
    const uint32_t all = uniform(place(off, groups, rows, log2, mult)) * tiles, each = (all + 7) / 8, at = b / 8, t = (b % 8) * each + at;
    if (at >= each || t >= all) return none;
    const uint32_t wanted = t / tiles;
    int from = 0, to = groups;
    while (to - from > 1) {
        const int apart = (to - from + 63) / 64, g = from + lane * apart;
        const uint64_t before = __ballot(g < to && place(off, g, rows, log2, mult) <= wanted);
        from += before ? (63 - __clzll((long long)before)) * apart : 0;
        to = to - from > apart ? from + apart : to;
    }
    int64_t lo, hi;
    const uint32_t count = uniform(group_chunks(off, from, groups, rows, log2, mult, empty, lo, hi)), first = uniform(place(off, from, rows, log2, mult));
    const uint32_t places = uniform(place(off, from + 1, rows, log2, mult)) - first;
    if (wanted < first || wanted - first >= places) return none;        // (in front of the first group, or offsets that fall)
    const uint32_t in_group = t - first * tiles, chunk = in_group % places;
    if (chunk >= count) return none;        // a place without a chunk
    lo = uniform64(lo);
    hi = uniform64(hi);
    const int64_t size = (int64_t)mult << log2, clo = lo + (int64_t)chunk * size, chi = clo + size;
    return {from, clo, chi < hi ? chi : hi, shared_place(lo, from, groups, rows, log2, mult) + chunk, count, in_group / places};
}

// Workgroup b's chunk and tile (of `tiles` that each chunk has).  All lanes of a wave together; the result is the same in every lane.
// `shared` is only found with `empty`, for sums.
// The chip's eight dies take workgroups in turn and have an L2 each, so die d gets the d-th eighth of the work, and within a group
// the chunks of one tile come one after the other: they read the same weights at about the same time.  A lane has a group.
__device__ __forceinline__ Chunk find_chunk(const int64_t* __restrict__ off, int groups, int64_t rows, int log2, uint32_t mult, uint32_t tiles, uint32_t b, bool empty) {
    if (groups > 64) return search_chunk(off, groups, rows, log2, mult, tiles, b, empty);
    const int lane = threadIdx.x & 63;
    int64_t lo, hi;
    const uint32_t n = group_chunks(off, lane, groups, rows, log2, mult, empty, lo, hi);
    const uint32_t sum = groups == 1 ? uniform(n) : wave_prefix(n);
    const uint32_t total = groups == 1 ? sum : (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    const uint32_t all = total * tiles, each = (all + 7) / 8, at = b / 8, t = (b % 8) * each + at;
    if (at >= each || t >= all) return {-1, 0, 0, 0, 0, 0};
    const int found = __ffsll((unsigned long long)__ballot(sum * tiles > t)) - 1;
    const int64_t glo = uniform64(__shfl(lo, found)), ghi = uniform64(__shfl(hi, found));
    const uint32_t count = uniform((uint32_t)__shfl((int)n, found)), first = uniform((uint32_t)__shfl((int)sum, found)) - count;
    const uint32_t in_group = t - first * tiles, chunk = tiles == 1 ? in_group : in_group % count;
    const int64_t size = (int64_t)mult << log2, clo = glo + (int64_t)chunk * size, chi = clo + size;
    const uint32_t shared = empty && groups > 1 ? wave_sum(n > 1 && lane < found ? n : 0) : 0;
    return {found, clo, chi < ghi ? chi : ghi, shared + chunk, count, tiles == 1 ? 0 : in_group / count};
}

}  // namespace pcc_train
