// Products of rows with the weights of their group, and their backward pass.
//
// Everything is one form of product, D[m][n] = sum_k P[m][k] Q[n][k], where m is the index that is contiguous in the
// result's memory:
//   forward    y[row][out] = x w^T      P = w  (m: out)   Q = x  (n: row)   k: in
//   backward   dx[row][in] = dz w       P = w^T (m: in)   Q = dz (n: row)   k: out
//   weights    dw[out][in] = dz^T x     P = x^T (m: in)   Q = dz^T (n: out) k: row
// v_mfma_f32_16x16x32: lane l gives P[m = l % 16][k = 8 (l / 16) ..+7] and Q[n = l % 16][same k] and gets
// D[m = 4 (l / 16) ..+3][n = l % 16], four neighbours of the result's memory.  An operand that has k contiguous in memory
// ("along") is read from LDS 16 bytes a lane; one that has its own index contiguous ("across") by ds_read_b64_tr_b16: of
// 16 lanes, lane j points at four values of row j / 4, column 4 (j % 4) and receives column j of the four rows.
#pragma once

#include "train_device.h"

namespace pcc_train {

struct Grouped {
    const u16* x;
    const u16* w;
    const u16* dz;
    const float* bias;
    const int64_t* off;
    void* y;            // forward: y; backward: dx
    float* dw;
    float* db;
    float* partial;     // weights: sums of one chunk, in * out + out values each
    size_t ldx, lddz, ldy;
    int64_t rows;
    int groups, in, out, act;
    int log2;           // rows of a chunk
    int y32;            // y is fp32
    uint32_t tiles_m, tiles_n;
};

constexpr int kTile = 128, kTileK = 64, kTileThreads = 256;

// An operand's tile in LDS, 16 KB.  Chunks of 8 values; chunk c of row r stands at slot c ^ swizzle(r) of the row, so that the
// rows that are read together lie in different banks.
//   along: rows are the operand's 128 indices, 64 k each (8 chunks)
//   across: rows are the 64 k, 128 indices each (16 chunks)
template <bool ACROSS>
struct TileLds {
    static constexpr int kChunks = ACROSS ? 16 : 8;
    __device__ static int at(int r, int c) { return (r * kChunks + (c ^ (ACROSS ? (2 * (r & 7)) : (r & 7)))) * 8; }
    // The MFMA operand of indices 16 i .. +15, k 32 kk .. +31.
    __device__ static u16x8 operand(const u16* lds, int i, int kk, int lane) {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const u16x8*>(lds + at(16 * i + (lane & 15), 4 * kk + (lane >> 4)));
        } else {
            u16x8 v;
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int r = 32 * kk + 8 * (lane >> 4) + ((lane & 15) >> 2), c = 2 * i + ((lane & 3) >> 1), e = 4 * (lane & 1);
            const u16x4 a = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r, c) + e)));
            const u16x4 b = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r + 4, c) + e)));
            for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[j + 4] = b[j]; }
            return v;
        }
    }
};

// Fill a tile from memory, zeros where there is nothing.  base is the value of index 0, k 0.
template <bool ACROSS>
__device__ __forceinline__ void stage(u16* lds, const u16* base, size_t ld, int64_t i0, int64_t ni, int64_t k0, int64_t nk) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int t = threadIdx.x + kTileThreads * s;
        const int r = t / TileLds<ACROSS>::kChunks, c = t % TileLds<ACROSS>::kChunks;
        const int64_t row = (ACROSS ? k0 : i0) + r, rows = ACROSS ? nk : ni;
        const int64_t col = (ACROSS ? i0 : k0) + 8 * c, cols = ACROSS ? ni : nk;
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < rows)
            for (int j = 0; j < 8; ++j)
                if (col + j < cols) v[j] = base[(size_t)row * ld + (size_t)(col + j)];
        *reinterpret_cast<u16x8*>(lds + TileLds<ACROSS>::at(r, c)) = v;
    }
}

enum Mode { kForward, kBackward, kWeights };

// Four waves, each 64 x 64 of the tile's 128 x 128.
template <class T, int MODE>
__global__ __launch_bounds__(kTileThreads) void grouped_tile_kernel(Grouped a) {
    constexpr bool kPAcross = MODE != kForward, kQAcross = MODE == kWeights;
    __shared__ __align__(16) u16 lds_p[kTile * kTileK], lds_q[kTile * kTileK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
    const uint32_t per_chunk = a.tiles_m * (MODE == kWeights ? a.tiles_n : 1);
    const uint32_t id = blockIdx.x / per_chunk, rest = blockIdx.x % per_chunk;
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, id, MODE == kWeights);
    if (ch.group < 0) return;
    const int64_t m0 = (int64_t)(rest % a.tiles_m) * kTile, n0 = MODE == kWeights ? (int64_t)(rest / a.tiles_m) * kTile : 0;
    const int64_t n_rows = ch.hi - ch.lo;
    const u16* w = a.w ? a.w + (size_t)ch.group * a.in * a.out : nullptr;
    const u16* p = MODE == kWeights ? a.x + (size_t)ch.lo * a.ldx : w;
    const u16* q = MODE == kForward ? a.x + (size_t)ch.lo * a.ldx : a.dz + (size_t)ch.lo * a.lddz;
    const size_t ldp = MODE == kWeights ? a.ldx : (size_t)a.in, ldq = MODE == kForward ? a.ldx : a.lddz;
    const int64_t np = MODE == kForward ? a.out : a.in, nq = MODE == kWeights ? a.out : n_rows;
    const int64_t nk = MODE == kForward ? a.in : MODE == kBackward ? a.out : n_rows;

    f32x4 acc[4][4] = {}, sums[4] = {};
    const bool with_db = MODE == kWeights && a.db && m0 == 0 && wm == 0;
    u16x8 ones;
    for (int j = 0; j < 8; ++j) ones[j] = T::kOne;
    for (int64_t k0 = 0; k0 < nk; k0 += kTileK) {
        stage<kPAcross>(lds_p, p, ldp, m0, np, k0, nk);
        stage<kQAcross>(lds_q, q, ldq, n0, nq, k0, nk);
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u16x8 fp[4], fq[4];
            for (int i = 0; i < 4; ++i) fp[i] = TileLds<kPAcross>::operand(lds_p, 4 * wm + i, kk, lane);
            for (int i = 0; i < 4; ++i) fq[i] = TileLds<kQAcross>::operand(lds_q, 4 * wn + i, kk, lane);
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(fp[i], fq[j], acc[i][j]);
            if (with_db)
                for (int j = 0; j < 4; ++j) sums[j] = T::mfma(ones, fq[j], sums[j]);
        }
        __syncthreads();
    }

    float* dw = nullptr;
    float* db = nullptr;
    if (MODE == kWeights) {
        const size_t size = (size_t)a.in * a.out;
        if (ch.count == 1) {
            dw = a.dw + (size_t)ch.group * size;
            db = a.db ? a.db + (size_t)ch.group * a.out : nullptr;
        } else {
            dw = a.partial + (size_t)id * (size + a.out);
            db = dw + size;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + 64 * wn + 16 * j + (lane & 15);
        if (n >= nq) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t m = m0 + 64 * wm + 16 * i + 4 * (lane >> 4) + e;
                if (m >= np) continue;
                float v = acc[i][j][e];
                if (MODE == kWeights) {
                    dw[(size_t)n * a.in + m] = v;
                } else {
                    const size_t at = (size_t)(ch.lo + n) * a.ldy + m;
                    if (MODE == kForward) v = activate(a.bias ? v + a.bias[(size_t)ch.group * a.out + m] : v, a.act);
                    else if (a.act != PCC_ACT_NONE) v = times_derivative(v, from16<T>(a.x[(size_t)(ch.lo + n) * a.ldx + m]), a.act);
                    if (a.y32) static_cast<float*>(a.y)[at] = v;
                    else static_cast<u16*>(a.y)[at] = to16<T>(v);
                }
            }
        }
        if (with_db && lane < 16) db[n] = sums[j][0];
    }
}

// Chunks' sums to those of their group, in the chunks' order.  A group of one chunk was written where it belongs.
__global__ __launch_bounds__(256) void grouped_reduce_kernel(Grouped a) {
    const int g = blockIdx.y;
    // the chunks of groups 0..g-1 come first: the chunk that a search for group g's first one finds
    const int lane = threadIdx.x & 63;
    uint32_t first = 0, count = 0;
    for (int g0 = 0; g0 <= g; g0 += 64) {
        const int i = g0 + lane;
        uint32_t n = 0;
        if (i <= g) {
            const int64_t lo = clamp64(a.off[i], 0, a.rows), hi = clamp64(a.off[i + 1], lo, a.rows);
            n = (uint32_t)((hi - lo + ((int64_t)1 << a.log2) - 1) >> a.log2);
            if (n == 0) n = 1;
        }
        if (i == g) count = n;
        for (int d = 32; d; d >>= 1) n += (uint32_t)__shfl_xor((int)n, d);
        first += n;
    }
    for (int d = 32; d; d >>= 1) count += (uint32_t)__shfl_xor((int)count, d);
    first -= count;
    if (count <= 1) return;
    const size_t size = (size_t)a.in * a.out, all = size + (a.db ? a.out : 0);
    for (size_t e = (size_t)blockIdx.x * blockDim.x + threadIdx.x; e < all; e += (size_t)gridDim.x * blockDim.x) {
        float s = 0.0f;
        for (uint32_t c = 0; c < count; ++c) s += a.partial[(size_t)(first + c) * (size + a.out) + e];
        if (e < size) a.dw[(size_t)g * size + e] = s;
        else a.db[(size_t)g * a.out + (e - size)] = s;
    }
}

}  // namespace pcc_train
