// Causal contexts as rows of network inputs.
//
// A lane has a pixel.  The bytes of its neighbours are three runs of memory (12 or 15 bytes of the two rows above, 6 of its own), which it
// loads by words; a value is a byte / 256, eight significant bits: exact in bf16.  The rows go through LDS, so that a wave
// writes its 64 rows 16 bytes a lane, neighbours next to each other: output is 20 to 27 times the input and sets the time:
// 24 pictures of 768x512, 12 neighbours, 202 us, 3.9 TB/s (a gather by bytes, 16 bytes of output a thread: 466).  The pictures are fetched
// 3.8 times, by the dies that have the rows above and the row itself: 4.3 TB/s in all.
#pragma once

#include "train_device.h"

namespace pcc_train {

struct Tap { int dr, dc; };
// Neighbour j of a pixel, in the order of the blob's first layer.
__host__ __device__ constexpr Tap tap_of(int nbhd, int delay, int j) {
    const int run = nbhd == 10 ? 4 : 5;
    Tap t = j < run ? Tap{-2, j - 2} : j < 2 * run ? Tap{-1, j - run - 2} : Tap{0, j - 2 * run - 2};
    // diagonal order: (r-2,c+2), (r-1,c+1), (r-1,c+2) are not decoded when (r,c) is; the pixel above stands in
    if (delay == 1 && ((t.dr == -2 && t.dc == 2) || (t.dr == -1 && t.dc >= 1))) t = {-1, 0};
    return t;
}

constexpr int kContextThreads = 256, kContextWidth = 40;

template <int NBHD, int DELAY>
__global__ __launch_bounds__(kContextThreads) void contexts_kernel(const uint8_t* __restrict__ img, uint64_t pixels, int H, int W, u16* __restrict__ x,
                                                                   int width, size_t ldx, int wide) {
    constexpr int kValues = 3 * NBHD, kChunks = kContextWidth / 8, kReach = NBHD == 10 ? 1 : 2;
    __shared__ __align__(16) u16x8 rows[kContextThreads / 64][64 * kChunks];        // five chunks a row: an odd distance
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t p0 = (uint64_t)blockIdx.x * kContextThreads + uniform(threadIdx.x & ~63u), p = p0 + lane;
    if (p0 >= pixels) return;
    const int n = pixels - p0 < 64 ? (int)(pixels - p0) : 64;
    const bool mine = lane < n;

    const uint64_t row0 = p0 / (uint32_t)W;
    const uint32_t along = (uint32_t)(p0 - row0 * (uint32_t)W) + lane, down = along / (uint32_t)W, c = along - down * (uint32_t)W;
    const uint32_t r = ((uint32_t)(row0 % (uint32_t)H) + down) % (uint32_t)H;
    // words of the runs from column c - 2 on: rows r - 2, r - 1, r
    uint32_t words[3][4] = {};
    const uint8_t* at = img + 3 * (int64_t)p;
    const int64_t pitch = 3 * (int64_t)W;
    if (mine && r >= 2 && c >= 2 && c + kReach < (uint32_t)W) {
        __builtin_memcpy(words[0], at - 2 * pitch - 6, 16);
        __builtin_memcpy(words[1], at - pitch - 6, 16);
        __builtin_memcpy(words[2], at - 6, 8);
    } else if (mine) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int i = 0; i < (k == 2 ? 6 : 3 * (kReach + 3)); ++i) {
                const int cc = (int)c + i / 3 - 2;
                if ((int)r + k >= 2 && cc >= 0 && cc < W) words[k][i / 4] |= (uint32_t)at[(k - 2) * pitch - 6 + i] << (8 * (i % 4));
            }
    }
    auto value = [&](int i) -> u16 {
        if (i >= kValues) return 0;
        const Tap t = tap_of(NBHD, DELAY, i / 3);
        const int byte = 3 * (t.dc + 2) + i % 3;
        return to16<Bf16>((float)((words[t.dr + 2][byte / 4] >> (8 * (byte % 4))) & 0xFFu) * (1.0f / 256.0f));
    };
    if (wide) {
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            u16x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = value(8 * k + e);
            rows[wave][lane * kChunks + k] = v;
        }
        __builtin_amdgcn_wave_barrier();
        typedef u16x8 at_four __attribute__((aligned(4)));
        const int chunks = width / 8;
        for (int id = lane; id < n * chunks; id += 64) {
            const int row = chunks == 5 ? id / 5 : id / 4, k = id - row * chunks;
            *reinterpret_cast<at_four*>(x + (p0 + row) * ldx + 8 * k) = rows[wave][row * kChunks + k];
        }
    } else if (mine) {
        u16* to = x + p * ldx;
#pragma unroll
        for (int i = 0; i < kValues; ++i) to[i] = value(i);
        for (int i = kValues; i < width; ++i) to[i] = 0;
    }
}

}  // namespace pcc_train
