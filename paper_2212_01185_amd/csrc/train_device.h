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
// every chunk of 2^log2 rows that could exist (rows / 2^log2, and one more a group for the parts), and a
// workgroup looks up which rows are its own.  Offsets are clamped to the rows there are and to rising order, so
// that wrong ones make wrong results but no access outside the tensors.
// ---------------------------------------------------------------------------
struct Chunk {
    int group;          // -1: there is no such chunk
    int64_t lo, hi;     // rows
    uint32_t first;     // number of the group's first chunk
    uint32_t count;     // chunks of the group
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    return (int64_t)(((uint64_t)uniform((uint32_t)((uint64_t)v >> 32)) << 32) | uniform((uint32_t)(uint64_t)v));
}

// All lanes of a wave together; the result is the same in every lane.  With `empty`, a group without rows has one chunk, of no rows.
__device__ __forceinline__ Chunk find_chunk(const int64_t* __restrict__ off, int groups, int64_t rows, int log2, uint32_t t, bool empty) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int g0 = 0; g0 < groups; g0 += 64) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        uint32_t n = 0;
        if (g < groups) {
            lo = clamp64(off[g], 0, rows);
            hi = clamp64(off[g + 1], lo, rows);
            n = (uint32_t)((hi - lo + ((int64_t)1 << log2) - 1) >> log2);
            if (empty && n == 0) n = 1;
        }
        uint32_t sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t up = (uint32_t)__shfl_up((int)sum, d);
            if (lane >= d) sum += up;
        }
        const uint64_t beyond = __ballot(before + sum > t);
        if (beyond) {
            const int at = __ffsll((unsigned long long)beyond) - 1;
            const int64_t glo = uniform64(__shfl(lo, at)), ghi = uniform64(__shfl(hi, at));
            const uint32_t count = uniform((uint32_t)__shfl((int)n, at)), first = before + uniform((uint32_t)__shfl((int)sum, at)) - count;
            const int64_t clo = glo + ((int64_t)(t - first) << log2);
            const int64_t chi = clo + ((int64_t)1 << log2);
            return {g0 + at, clo, chi < ghi ? chi : ghi, first, count};
        }
        before += uniform((uint32_t)__shfl((int)sum, 63));
    }
    return {-1, 0, 0, 0, 0};
}

}  // namespace pcc_train
