// AdamW over many tensors.
//
// One launch for all: a list of pieces of 4,096 elements (1,024 where there are few), made when the plan is, says which tensor a
// workgroup works on.  Every
// element is read once and written once: 16 + 12 bytes with states in 32 bits, 10 + 6 in 8 bits, and what the copy takes.  33.5 million
// elements with a bf16 copy: 205 us with 32 bits (4.9 TB/s, memory), 166 with 8 (3.6 TB/s, and the vector ALU busy for 57 % of the time: a
// wave's loads, then exact roots and codes, exchanges and stores come one after the other, so neither is full).
//
// 8-bit states.  A wave has a block of 256 elements, four a lane, and finds its largest magnitudes by exchanges.  Codes are e4m3: a
// step of a code is 1/8 to 1/16 of the value, and one step of the second moment's average changes it by 1 - beta2, a
// thousandth: to the nearest it would stay where it is for good.  So a code is cut, not rounded, after a part of its step was
// added that runs through all parts evenly over the steps (a mix of the place in the block and the step's number): the mean
// over the steps is the value.
#pragma once

#include <type_traits>

#include "train_device.h"

namespace pcc_train {

struct AdamwTensor {
    float* param;
    const void* grad;
    u16* copy;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    uint64_t n;
    uint32_t aligned;       // four elements at a time can be read and written in one piece
    uint32_t unused;
};
struct AdamwPiece {
    uint32_t tensor, part;
};
constexpr int kAdamwThreads = 256;
constexpr int kStateBlock = 256;
// Blocks of a wave in a piece.  One where all pieces of four would not fill the chip (505,000 elements).
constexpr int piece_blocks(uint64_t elements) { return elements < ((uint64_t)1 << 22) ? 1 : 4; }
constexpr uint64_t piece_elements(int blocks) { return (uint64_t)blocks * (kAdamwThreads / 64) * kStateBlock; }

// What a step's number makes of the hyperparameters; written by a kernel of one thread in front of the step's.
struct AdamwRates {
    float rate, root, keep;
    uint32_t t;
};

struct AdamwArgs {
    const AdamwTensor* tensors;
    const AdamwPiece* pieces;
    uint32_t n_pieces;
    int piece_blocks;
    const AdamwRates* rates;
    float b1, rest1, b2, rest2, eps;
};

// b^t for t >= 0 by squaring.
__device__ __forceinline__ double power(double b, uint64_t t) {
    double r = 1.0;
    for (; t; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}

// The part of a code's step (20 bits) that place i of a block adds at step t; the second moment's is another mix.
__device__ __forceinline__ uint32_t dither_bits(uint32_t i, uint32_t t) {
    uint32_t h = i * 0x9E3779B9u + t * 0xB7E15163u;
    h ^= h >> 15;
    h *= 0x6A09E667u;
    h ^= h >> 13;
    h *= 0x9E3779B9u;
    h ^= h >> 16;
    return h;
}

// e4m3 code of y, 0 <= y <= 448, after `part` / 2^20 of a step: bits from the exponent on, or eighths of 2^-6 below it.
__device__ __forceinline__ uint32_t code_of(float y, uint32_t part) {
    if (!(y <= 1e30f)) return 0x7Fu;      // not a number, or infinite: the code of NaN
    const uint32_t normal = ((__builtin_bit_cast(uint32_t, y) + part) >> 20) - (120u << 3);
    const uint32_t small = (uint32_t)(y * 512.0f + (float)part * 0x1p-20f);
    const uint32_t code = y >= 0x1p-6f ? normal : small;
    return code < 0x7Eu ? code : 0x7Eu;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// Four elements of a tensor from element i on, `n` of them there (zeros for the others): in one piece if they can be.
template <class V, class E>
__device__ __forceinline__ V load_four(const E* from, uint64_t i, int n, bool wide) {
    if (wide) return *reinterpret_cast<const V*>(from + i);
    V v = {};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) v[j] = from[i + j];
    return v;
}
template <class V, class E>
__device__ __forceinline__ void save_four(E* to, uint64_t i, V v, int n, bool wide) {
    if (wide) { *reinterpret_cast<V*>(to + i) = v; return; }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) to[i + j] = v[j];
}
// Four codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* from, uint64_t i, int n, bool wide) {
    if (wide) return *reinterpret_cast<const uint32_t*>(from + i);
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) word |= (uint32_t)from[i + j] << (8 * j);
    return word;
}
__device__ __forceinline__ void save_codes(uint8_t* to, uint64_t i, uint32_t word, int n, bool wide) {
    if (wide) { *reinterpret_cast<uint32_t*>(to + i) = word; return; }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < n) to[i + j] = (uint8_t)(word >> (8 * j));
}
__device__ __forceinline__ f32x4 values_of(uint32_t word) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
    return {a[0], a[1], b[0], b[1]};
}
template <int GRAD>
__device__ __forceinline__ f32x4 load_gradient(const void* g, uint64_t i, int n, bool wide) {
    if constexpr (GRAD == PCC_FP32) {
        return load_four<f32x4>(static_cast<const float*>(g), i, n, wide);
    } else {
        using T = std::conditional_t<GRAD == PCC_BF16, Bf16, Fp16>;
        const u16x4 v = load_four<u16x4>(static_cast<const u16*>(g), i, n, wide);
        return {from16<T>(v[0]), from16<T>(v[1]), from16<T>(v[2]), from16<T>(v[3])};
    }
}

// A wave's block of 256 elements.  (The next block's loads before this one's step gained nothing on many elements and cost few dearly: twice the
// code, which a wave runs once; 505,000 elements, 8 bits, 20.9 us with and 9.9 without.)
template <int GRAD, int COPY, int BITS>
struct AdamwBlock {
    f32x4 p, g, m, v;
    uint32_t mc, vc;
    float ms, vs;
    uint64_t block, i;
    int n;          // of this lane's four elements
    bool wide;

    __device__ void load(const AdamwTensor& s, uint64_t b, int lane) {
        block = b;
        i = b * kStateBlock + 4 * lane;
        n = i >= s.n ? 0 : s.n - i < 4 ? (int)(s.n - i) : 4;
        wide = s.aligned && n == 4;
        p = load_four<f32x4>(s.param, i, n, wide);
        g = load_gradient<GRAD>(s.grad, i, n, wide);
        if constexpr (BITS == 32) {
            m = load_four<f32x4>(static_cast<const float*>(s.m), i, n, wide);
            v = load_four<f32x4>(static_cast<const float*>(s.v), i, n, wide);
        } else {
            mc = load_codes(static_cast<const uint8_t*>(s.m), i, n, wide);
            vc = load_codes(static_cast<const uint8_t*>(s.v), i, n, wide);
            ms = s.m_scale[b];
            vs = s.v_scale[b];
        }
    }
    __device__ void step(const AdamwTensor& s, const AdamwArgs& a, const AdamwRates& k, const uint32_t (&mix)[4], int lane) {
        if constexpr (BITS == 8) {
            m = values_of(mc) * ms;
            v = values_of(vc) * vs;
            v = v * v;
        }
        f32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m[j] = a.b1 * m[j] + a.rest1 * g[j];
            v[j] = a.b2 * v[j] + (a.rest2 * g[j]) * g[j];
            r[j] = sqrtf(v[j]);
            // the quotient by the reciprocal's hardware approximation and a product: 1.5 steps of fp32 off at most, on an update that is a
            // small part of the parameter
            p[j] = p[j] * k.keep - k.rate * (m[j] * __builtin_amdgcn_rcpf(r[j] * k.root + a.eps));
        }
        save_four(s.param, i, p, n, wide);
        if (s.copy) {
            using T = std::conditional_t<COPY == PCC_BF16, Bf16, Fp16>;
            save_four(s.copy, i, u16x4{to16<T>(p[0]), to16<T>(p[1]), to16<T>(p[2]), to16<T>(p[3])}, n, wide);
        }
        if constexpr (BITS == 32) {
            save_four(static_cast<float*>(s.m), i, m, n, wide);
            save_four(static_cast<float*>(s.v), i, v, n, wide);
        } else {
            float mmax = 0.0f, rmax = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mmax = fmaxf(mmax, j < n ? fabsf(m[j]) : 0.0f);
                rmax = fmaxf(rmax, j < n ? r[j] : 0.0f);
            }
            mmax = wave_max(mmax);
            rmax = wave_max(rmax);
            if (mmax == INFINITY || rmax == INFINITY) {     // an infinite scale would make every other code of the block 0 * inf
                mmax = rmax = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    mmax = fmaxf(mmax, j < n && fabsf(m[j]) < INFINITY ? fabsf(m[j]) : 0.0f);
                    rmax = fmaxf(rmax, j < n && r[j] < INFINITY ? r[j] : 0.0f);
                }
                mmax = wave_max(mmax);
                rmax = wave_max(rmax);
            }
            const float msc = mmax * (1.0f / 448.0f), rsc = rmax * (1.0f / 448.0f);
            const float minv = msc >= 0x1p-100f ? 1.0f / msc : 0.0f, rinv = rsc >= 0x1p-100f ? 1.0f / rsc : 0.0f;
            uint32_t new_m = 0, new_v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = mix[j];
                const uint32_t cm = code_of(fabsf(m[j]) * minv, h >> 12), cv = code_of(r[j] * rinv, (h * 0xB7E15163u) >> 12);
                new_m |= (cm | (m[j] < 0.0f ? 0x80u : 0u)) << (8 * j);
                new_v |= (r[j] > 0.0f && cv == 0 ? 1u : cv) << (8 * j);
            }
            save_codes(static_cast<uint8_t*>(s.m), i, new_m, n, wide);
            save_codes(static_cast<uint8_t*>(s.v), i, new_v, n, wide);
            if (lane == 0) { s.m_scale[block] = msc; s.v_scale[block] = rsc; }
        }
    }
};

template <int GRAD, int COPY, int BITS>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AdamwRates k = *a.rates;
    uint32_t mix[4];
    for (int j = 0; j < 4; ++j) mix[j] = BITS == 8 ? dither_bits((uint32_t)(4 * lane + j), k.t) : 0;
    for (uint32_t at = blockIdx.x; at < a.n_pieces; at += gridDim.x) {
        const AdamwPiece piece = a.pieces[at];
        const AdamwTensor s = a.tensors[piece.tensor];
        const uint64_t first = ((uint64_t)piece.part * (kAdamwThreads / 64) + wave) * a.piece_blocks, blocks = (s.n + kStateBlock - 1) / kStateBlock;
        const uint64_t end = first + a.piece_blocks < blocks ? first + a.piece_blocks : blocks;
        for (uint64_t j = first; j < end; ++j) {
            AdamwBlock<GRAD, COPY, BITS> one;
            one.load(s, j, lane);
            one.step(s, a, k, mix, lane);
        }
    }
}

// A kernel of its own, some 2 us: else every workgroup of the step would take two powers in 64 bits, and the last one would have to be found
// to write the step's number.
__global__ void adamw_prepare_kernel(int64_t* step, const float* d_lr, double lr, double beta1, double beta2, double weight_decay, AdamwRates* to) {
    const int64_t t = *step + 1;
    if (d_lr) lr = (double)*d_lr;
    *to = {(float)(lr / (1.0 - power(beta1, (uint64_t)t))), (float)(1.0 / sqrt(1.0 - power(beta2, (uint64_t)t))), (float)(1.0 - lr * weight_decay), (uint32_t)t};
    *step = t;
}

}  // namespace pcc_train
