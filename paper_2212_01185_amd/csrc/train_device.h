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

// Workgroup b's chunk and tile (of `tiles` that each chunk has).  All lanes of a wave together; the result is the same in every lane.
// `shared` is only found with `empty`, for sums.
// The chip's eight dies take workgroups in turn and have an L2 each, so die d gets the d-th eighth of the work, and within a group
// the chunks of one tile come one after the other: they read the same weights at about the same time.
__device__ __forceinline__ Chunk find_chunk(const int64_t* __restrict__ off, int groups, int64_t rows, int log2, uint32_t mult, uint32_t tiles, uint32_t b, bool empty) {
    const int lane = threadIdx.x & 63;
    uint32_t total = 0;
    if (groups > 64) {                  // else the search itself says it
        for (int g0 = 0; g0 < groups; g0 += 64) {
            int64_t lo, hi;
            total += wave_sum(group_chunks(off, g0 + lane, groups, rows, log2, mult, empty, lo, hi));
        }
    }
    uint32_t before = 0, shared = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        int64_t lo, hi;
        const uint32_t n = group_chunks(off, g0 + lane, groups, rows, log2, mult, empty, lo, hi);
        const uint32_t sum = groups == 1 ? uniform(n) : wave_prefix(n);
        if (groups <= 64) total = groups == 1 ? sum : (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
        const uint32_t all = total * tiles, each = (all + 7) / 8, at = b / 8, t = (b % 8) * each + at;
        if (at >= each || t >= all) break;
        const uint64_t beyond = __ballot((before + sum) * tiles > t);
        if (beyond) {
            const int found = __ffsll((unsigned long long)beyond) - 1;
            const int64_t glo = uniform64(__shfl(lo, found)), ghi = uniform64(__shfl(hi, found));
            const uint32_t count = uniform((uint32_t)__shfl((int)n, found)), first = before + uniform((uint32_t)__shfl((int)sum, found)) - count;
            const uint32_t in_group = t - first * tiles, chunk = tiles == 1 ? in_group : in_group % count;
            const int64_t size = (int64_t)mult << log2, clo = glo + (int64_t)chunk * size, chi = clo + size;
            if (empty && groups > 1) shared += wave_sum(n > 1 && lane < found ? n : 0);
            return {g0 + found, clo, chi < ghi ? chi : ghi, shared + chunk, count, tiles == 1 ? 0 : in_group / count};
        }
        before += uniform((uint32_t)__shfl((int)sum, 63));
        if (empty) shared += wave_sum(n > 1 ? n : 0);
    }
    return {-1, 0, 0, 0, 0, 0};
}

}  // namespace pcc_train
