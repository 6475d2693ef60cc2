// AdamW over many tensors.
//
// One launch for all: a list of pieces of 4,096 elements, made when the plan is, says which tensor a workgroup works on.  Every
// element is read once and written once: 16 + 12 bytes with states in 32 bits, 10 + 6 in 8 bits, and what the copy takes.
//
// 8-bit states.  A wave has a block of 256 elements, four a lane, and finds its largest magnitudes by exchanges.  Codes are e4m3: a
// step of a code is 1/8 to 1/16 of the value, and one step of the second moment's average changes it by 1 - beta2, a
// thousandth: to the nearest it would stay where it is for good.  So a code is cut, not rounded, after a part of its step was
// added that runs through all parts evenly over the steps (a mix of the place in the block and the step's number): the mean
// over the steps is the value.
#pragma once

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
constexpr int kPiece = 4096, kAdamwThreads = 256;
constexpr int kStateBlock = 256;

struct AdamwArgs {
    const AdamwTensor* tensors;
    const AdamwPiece* pieces;
    uint32_t n_pieces;
    uint32_t* ticket;
    int64_t* step;
    const float* d_lr;
    double lr, beta1, beta2, weight_decay;
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
    if (!(y <= 1e30f)) return 0x7Fu;      // not a number: its own code
    const uint32_t normal = ((__builtin_bit_cast(uint32_t, y) + part) >> 20) - (120u << 3);
    const uint32_t small = (uint32_t)(y * 512.0f + (float)part * 0x1p-20f);
    const uint32_t code = y >= 0x1p-6f ? normal : small;
    return code < 0x7Eu ? code : 0x7Eu;
}
__device__ __forceinline__ float value_of(uint32_t code) {
    const uint32_t e = (code >> 3) & 15u, f = code & 7u;
    if ((code & 0x7Fu) == 0x7Fu) return __builtin_nanf("");
    const float v = e ? __builtin_bit_cast(float, ((e + 120u) << 23) | (f << 20)) : (float)f * 0x1p-9f;
    return code & 0x80u ? -v : v;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

template <int GRAD>
__device__ __forceinline__ float gradient(const void* g, uint64_t i) {
    if (GRAD == PCC_FP32) return static_cast<const float*>(g)[i];
    const u16 v = static_cast<const u16*>(g)[i];
    return GRAD == PCC_BF16 ? from16<Bf16>(v) : from16<Fp16>(v);
}

template <int GRAD, int COPY, int BITS>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(AdamwArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = *a.step + 1;
    const double lr = a.d_lr ? (double)*a.d_lr : a.lr;
    const float rate = (float)(lr / (1.0 - power(a.beta1, (uint64_t)t))), root = (float)(1.0 / sqrt(1.0 - power(a.beta2, (uint64_t)t)));
    const float keep = (float)(1.0 - lr * a.weight_decay);
    for (uint32_t at = blockIdx.x; at < a.n_pieces; at += gridDim.x) {
        const AdamwPiece piece = a.pieces[at];
        const AdamwTensor& s = a.tensors[piece.tensor];
        for (int b = wave; b < kPiece / kStateBlock; b += kAdamwThreads / 64) {
            const uint64_t block = (uint64_t)piece.part * (kPiece / kStateBlock) + b, i0 = block * kStateBlock + 4 * lane;
            if (block * kStateBlock >= s.n) break;
            float p[4], g[4], m[4], v[4], r[4];
            const float ms = BITS == 8 ? s.m_scale[block] : 0.0f, vs = BITS == 8 ? s.v_scale[block] : 0.0f;
            float mmax = 0.0f, rmax = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t i = i0 + j;
                m[j] = v[j] = r[j] = 0.0f;
                if (i >= s.n) continue;
                p[j] = s.param[i];
                g[j] = gradient<GRAD>(s.grad, i);
                if (BITS == 32) {
                    m[j] = static_cast<const float*>(s.m)[i];
                    v[j] = static_cast<const float*>(s.v)[i];
                } else {
                    m[j] = value_of(static_cast<const uint8_t*>(s.m)[i]) * ms;
                    v[j] = value_of(static_cast<const uint8_t*>(s.v)[i]) * vs;
                    v[j] = v[j] * v[j];
                }
                m[j] = a.b1 * m[j] + a.rest1 * g[j];
                v[j] = a.b2 * v[j] + (a.rest2 * g[j]) * g[j];
                r[j] = sqrtf(v[j]);
                p[j] = p[j] * keep - rate * (m[j] / (r[j] * root + a.eps));
                s.param[i] = p[j];
                if (s.copy) s.copy[i] = COPY == PCC_BF16 ? to16<Bf16>(p[j]) : to16<Fp16>(p[j]);
                if (BITS == 32) {
                    static_cast<float*>(s.m)[i] = m[j];
                    static_cast<float*>(s.v)[i] = v[j];
                }
                mmax = fmaxf(mmax, fabsf(m[j]));
                rmax = fmaxf(rmax, r[j]);
            }
            if (BITS == 8) {
                const float msc = wave_max(mmax) * (1.0f / 448.0f), rsc = wave_max(rmax) * (1.0f / 448.0f);
                const float minv = msc >= 0x1p-100f ? 1.0f / msc : 0.0f, rinv = rsc >= 0x1p-100f ? 1.0f / rsc : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint64_t i = i0 + j;
                    if (i >= s.n) continue;
                    const uint32_t h = dither_bits((uint32_t)(4 * lane + j), (uint32_t)t);
                    const uint32_t cm = code_of(fabsf(m[j]) * minv, h >> 12), cv = code_of(r[j] * rinv, (h * 0xB7E15163u) >> 12);
                    static_cast<uint8_t*>(s.m)[i] = (uint8_t)(cm | (m[j] < 0.0f ? 0x80u : 0u));
                    static_cast<uint8_t*>(s.v)[i] = (uint8_t)(r[j] > 0.0f && cv == 0 ? 1u : cv);
                }
                if (lane == 0) { s.m_scale[block] = msc; s.v_scale[block] = rsc; }
            }
        }
    }
    // the last workgroup to come here writes the step's number: all have read it
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(a.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == gridDim.x - 1) {
            *a.step = t;
            __hip_atomic_store(a.ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
}

}  // namespace pcc_train
