// Dropout whose mask is never stored: y = residual + x / (1 - p) where an element is kept, residual where it is not.
//
// An element's 16 random bits are a function of the seed, the step, its row and its column: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw,
// Parallel random numbers: as easy as 1, 2, 3, 2011), whose counter is (column / 8 | bits 32.. of the row << 16, row, step) and whose
// key is the seed; its 128 bits are those of eight neighbours.  So the backward pass makes the same mask again, and strides, types and launches do
// not matter.  An element is dropped if its bits are below round(65536 p).
#pragma once

#include "train_rows.h"

namespace pcc_train {

struct Dropout {
    const void* x;
    const void* residual;   // or null: 0
    void* y;
    size_t ldx, ldr, ldy;
    uint64_t rows, seed;
    const int64_t* step;    // or null: 0
    uint32_t border;        // of 65536
    float scale;
    int features;
    uint32_t chunks;        // eights of a row
};

struct Philox {
    uint32_t c[4];
};
__device__ __forceinline__ Philox philox(Philox s, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * s.c[0], b = (uint64_t)0xCD9E8D57u * s.c[2];
        s = {{(uint32_t)(b >> 32) ^ s.c[1] ^ k0, (uint32_t)b, (uint32_t)(a >> 32) ^ s.c[3] ^ k1, (uint32_t)a}};
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return s;
}

constexpr int kDropoutThreads = 256;

// A thread has eight neighbours of a row: their bits are one turn of the generator.  With 16 bits an element its multiplications fit beside the loads:
// 16,384 rows of 4,096 in bf16 with a residual 70 us, 5.7 TB/s, the vector ALU busy for 58 % of it (bits of 32 would take twice as many turns).
template <class X, class Y>
__global__ __launch_bounds__(kDropoutThreads) void dropout_kernel(Dropout a) {
    const uint64_t id = (uint64_t)blockIdx.x * kDropoutThreads + threadIdx.x, row = id / a.chunks;
    if (row >= a.rows) return;
    const uint32_t chunk = (uint32_t)(id - row * a.chunks);
    const int f = 8 * (int)chunk;
    const uint64_t step = a.step ? (uint64_t)*a.step : 0;
    Eight<X> x;
    Eight<Y> y;
    x.load(a.x, row * a.ldx + f, a.features - f);
    if (a.residual) y.load(a.residual, row * a.ldr + f, a.features - f);
    const Philox bits = philox({{chunk | (uint32_t)(row >> 32) << 16, (uint32_t)row, (uint32_t)step, (uint32_t)(step >> 32)}}, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    float out[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool kept = ((bits.c[e / 2] >> (16 * (e & 1))) & 0xFFFFu) >= a.border;
        const float v = kept ? x.get(e) * a.scale : 0.0f;
        out[e] = a.residual ? y.get(e) + v : v;
    }
    y.set(out);
    y.store(a.y, row * a.ldy + f, a.features - f);
}

}  // namespace pcc_train
