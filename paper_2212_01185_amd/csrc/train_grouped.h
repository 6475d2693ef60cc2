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
    int log2;           // rows of a chunk: mult * 2^log2
    uint32_t mult;
    int y32;            // y is fp32
    int staged;         // forward, narrow: outputs go through LDS
    int wide_out, wide_x, wide_dw;  // four values of a row of the result, of x, of dw can be stored, read in one piece
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

typedef __attribute__((address_space(3))) void lds_void;

// An operand in memory, and a workgroup's way through it in steps of 64 k.  Where rows begin at even elements (`wide`), chunks go from
// memory to LDS without a register, 16 bytes a lane; a chunk that is cut by the end of its row is read value by value, and what lies
// beyond the operand is zero: such a lane's offset is beyond the buffer's end, for which the load gives zeros.  Rows at
// odd elements are read value by value.
template <bool ACROSS>
struct Source {
    const u16* base;            // index i0, k 0
    size_t ld;
    int64_t ni, nk;             // indices from i0 on, all k
    uint32_t offset[4];         // bytes of this lane's chunks from base + the step
    static constexpr uint32_t kNone = 0x7FFFFF00u;      // beyond the buffer (rows are at most 2^22 values, a tile has 128)

    __device__ void init(const u16* b, size_t stride, int64_t i0, int64_t n_index, int64_t n_k) {
        base = b + (ACROSS ? (size_t)i0 : (size_t)i0 * stride);
        ld = stride;
        ni = n_index - i0;
        nk = n_k;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            int r, c;
            place(s, r, c);
            const bool there = ACROSS ? 8 * c < ni : r < ni;
            offset[s] = there ? (uint32_t)(((size_t)r * ld + 8 * c) * 2) : kNone;
        }
    }
    __device__ static void place(int s, int& r, int& c) {
        const int slot = threadIdx.x + kTileThreads * s;
        r = slot / TileLds<ACROSS>::kChunks;
        c = (slot % TileLds<ACROSS>::kChunks) ^ (ACROSS ? 2 * (r & 7) : (r & 7));
    }
    // Values of a chunk that are there, at k0.
    __device__ int values(int r, int c, int64_t k0) const {
        const int64_t n = ACROSS ? (k0 + r < nk ? ni - 8 * c : 0) : (r < ni ? nk - k0 - 8 * c : 0);
        return n < 0 ? 0 : n > 8 ? 8 : (int)n;
    }
    __device__ void one_by_one(u16* lds, int s, int64_t k0, int n) const {
        int r, c;
        place(s, r, c);
        const u16* from = base + (ACROSS ? (size_t)(k0 + r) * ld + 8 * c : (size_t)r * ld + (size_t)k0 + 8 * c);
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) v[j] = from[j];
        *reinterpret_cast<u16x8*>(lds + (threadIdx.x + kTileThreads * s) * 8) = v;
    }
    template <bool WIDE>
    __device__ void stage(u16* lds, int64_t k0) const {
        if constexpr (!WIDE) {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                int r, c;
                place(s, r, c);
                one_by_one(lds, s, k0, values(r, c, k0));
            }
        } else {
            const __amdgpu_buffer_rsrc_t from =
                __builtin_amdgcn_make_buffer_rsrc((void*)(base + (ACROSS ? (size_t)k0 * ld : (size_t)k0)), 0, (int)kNone, 0x00020000);
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            const bool whole = k0 + kTileK <= nk && (!ACROSS || ni % 8 == 0 || ni >= kTile);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                lds_void* to = (lds_void*)(lds + (64 * wave + kTileThreads * s) * 8);
                if (whole) {
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to, 16, offset[s], 0, 0, 0);
                } else {
                    int r, c;
                    place(s, r, c);
                    const int n = values(r, c, k0);
                    if (n == 0 || n == 8) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to, 16, n ? offset[s] : kNone, 0, 0, 0);
                    else one_by_one(lds, s, k0, n);
                }
            }
        }
    }
};

// Values of a chunk's sums in the workspace: dw, db, and up to a multiple of four.
__host__ __device__ constexpr size_t partial_values(int in, int out) { return ((size_t)in * out + out + 3) / 4 * 4; }

enum Mode { kForward, kBackward, kWeights };

__device__ __forceinline__ void store_four(float* to, f32x4 v, int left, bool wide) {
    if (wide && left == 4) { *reinterpret_cast<f32x4*>(to) = v; return; }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) to[e] = v[e];
}

// Bias and activation, or the activation's derivative, of four neighbouring results of a row, and their store.
template <class T, int MODE>
__device__ __forceinline__ void finish_four(const Grouped& a, int group, size_t row, int64_t m, f32x4 v, int left) {
    const bool wide = a.wide_out && left == 4;
    if (MODE == kForward) {
        if (a.bias) {
            const float* bias = a.bias + (size_t)group * a.out + m;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += bias[e < left ? e : 0];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = activate(v[e], a.act);
    } else if (a.act != PCC_ACT_NONE) {
        const u16* x = a.x + row * a.ldx + m;
        u16x4 s = {0, 0, 0, 0};
        if (a.wide_x && left == 4) s = *reinterpret_cast<const u16x4*>(x);
        else for (int e = 0; e < 4; ++e) if (e < left) s[e] = x[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = times_derivative(v[e], from16<T>(s[e]), a.act);
    }
    const size_t at = row * a.ldy + m;
    if (a.y32) { store_four(static_cast<float*>(a.y) + at, v, left, wide); return; }
    u16x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = to16<T>(v[e]);
    u16* y = static_cast<u16*>(a.y) + at;
    if (wide) *reinterpret_cast<u16x4*>(y) = o;
    else for (int e = 0; e < 4; ++e) if (e < left) y[e] = o[e];
}

// Eight neighbouring results of a row after the activation, `left` of them there.
template <class T>
__device__ __forceinline__ void store_eight(const Grouped& a, size_t at, f32x4 v0, f32x4 v1, int left, int act) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v0[e] = activate(v0[e], act); v1[e] = activate(v1[e], act); }
    if (a.y32) {
        float* y = static_cast<float*>(a.y) + at;
        store_four(y, v0, left < 4 ? left : 4, a.wide_out);
        if (left > 4) store_four(y + 4, v1, left < 8 ? left - 4 : 4, a.wide_out);
        return;
    }
    u16x8 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) { o[e] = to16<T>(v0[e]); o[4 + e] = to16<T>(v1[e]); }
    u16* y = static_cast<u16*>(a.y) + at;
    if (a.wide_out && left >= 8) *reinterpret_cast<u16x8*>(y) = o;
    else
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) y[e] = o[e];
}

// Four waves, each 64 x 64 of the tile's 128 x 128.  Two tiles in LDS for each operand: the next step's is filled while this one's is
// multiplied.
template <class T, int MODE, bool WIDE>
__global__ __launch_bounds__(kTileThreads, 2) void grouped_tile_kernel(Grouped a) {
    constexpr bool kPAcross = MODE != kForward, kQAcross = MODE == kWeights;
    __shared__ __align__(16) u16 lds[2][2][kTile * kTileK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
    const uint32_t tiles = a.tiles_m * (MODE == kWeights ? a.tiles_n : 1);
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, tiles, blockIdx.x, MODE == kWeights);
    if (ch.group < 0) return;
    const int64_t m0 = (int64_t)(ch.part % a.tiles_m) * kTile, n0 = MODE == kWeights ? (int64_t)(ch.part / a.tiles_m) * kTile : 0;
    const int64_t n_rows = ch.hi - ch.lo;
    const u16* w = a.w ? a.w + (size_t)ch.group * a.in * a.out : nullptr;
    const int64_t np = MODE == kForward ? a.out : a.in, nq = MODE == kWeights ? a.out : n_rows;
    const int64_t nk = MODE == kForward ? a.in : MODE == kBackward ? a.out : n_rows;
    Source<kPAcross> p;
    Source<kQAcross> q;
    p.init(MODE == kWeights ? a.x + (size_t)ch.lo * a.ldx : w, MODE == kWeights ? a.ldx : (size_t)a.in, m0, np, nk);
    if (MODE == kForward) q.init(a.x + (size_t)ch.lo * a.ldx, a.ldx, n0, nq, nk);
    else q.init(a.dz + (size_t)ch.lo * a.lddz, a.lddz, n0, nq, nk);

    f32x4 acc[4][4] = {}, sums[4] = {};
    const bool with_db = MODE == kWeights && a.db && m0 == 0 && wm == 0;
    u16x8 ones;
    for (int j = 0; j < 8; ++j) ones[j] = T::kOne;
    if (nk > 0) {
        p.template stage<WIDE>(lds[0][0], 0);
        q.template stage<WIDE>(lds[0][1], 0);
    }
    int now = 0;
    for (int64_t k0 = 0; k0 < nk; k0 += kTileK, now ^= 1) {
        __builtin_amdgcn_s_waitcnt(0);      // this step's chunks are in LDS: the barrier alone does not wait for loads that go there
        __syncthreads();
        if (k0 + kTileK < nk) {
            p.template stage<WIDE>(lds[now ^ 1][0], k0 + kTileK);
            q.template stage<WIDE>(lds[now ^ 1][1], k0 + kTileK);
        }
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            u16x8 fp[4], fq[4];
            for (int i = 0; i < 4; ++i) fp[i] = TileLds<kPAcross>::operand(lds[now][0], 4 * wm + i, kk, lane);
            for (int i = 0; i < 4; ++i) fq[i] = TileLds<kQAcross>::operand(lds[now][1], 4 * wn + i, kk, lane);
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(fp[i], fq[j], acc[i][j]);
            if (with_db)
                for (int j = 0; j < 4; ++j) sums[j] = T::mfma(ones, fq[j], sums[j]);
        }
    }

    float* dw = nullptr;
    float* db = nullptr;
    if (MODE == kWeights) {
        const size_t size = (size_t)a.in * a.out;
        if (ch.count == 1) {
            dw = a.dw + (size_t)ch.group * size;
            db = a.db ? a.db + (size_t)ch.group * a.out : nullptr;
        } else {
            dw = a.partial + (size_t)ch.id * partial_values(a.in, a.out);
            db = dw + size;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + 64 * wn + 16 * j + (lane & 15);
        if (n >= nq) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t m = m0 + 64 * wm + 16 * i + 4 * (lane >> 4);
            const int left = np - m >= 4 ? 4 : (int)(np - m);
            if (left <= 0) continue;
            if (MODE == kWeights) store_four(dw + (size_t)n * a.in + m, acc[i][j], left, a.in % 4 == 0 && a.wide_dw);
            else finish_four<T, MODE>(a, ch.group, (size_t)(ch.lo + n), m, acc[i][j], left);
        }
        if (with_db && lane < 16) db[n] = sums[j][0];
    }
}

// Chunks' sums to those of their group, always in the same order.  A group of one chunk was written where it belongs.  A workgroup has 64
// values; 16 slices of its threads sum every 16th chunk, so that as many loads are on their way, then the slices are summed.
__global__ __launch_bounds__(256) void grouped_reduce_kernel(Grouped a) {
    __shared__ __align__(16) f32x4 slices[16][16];
    const int g = blockIdx.y, lane = threadIdx.x & 63;
    uint32_t first = 0, count = 0;
    for (int g0 = 0; g0 <= g; g0 += 64) {
        int64_t lo, hi;
        uint32_t n = group_chunks(a.off, g0 + lane, g + 1, a.rows, a.log2, a.mult, true, lo, hi);
        if (g0 + lane == g) count = n;
        for (int d = 32; d; d >>= 1) n += (uint32_t)__shfl_xor((int)n, d);
        first += n;
    }
    for (int d = 32; d; d >>= 1) count += (uint32_t)__shfl_xor((int)count, d);
    first -= count;
    if (count <= 1) return;
    const size_t size = (size_t)a.in * a.out, all = size + a.out, stride = partial_values(a.in, a.out);
    const int quad = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const size_t e0 = (size_t)blockIdx.x * 64 + 4 * quad;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (e0 < all) {
        const float* from = a.partial + (size_t)first * stride + e0;
#pragma unroll 4
        for (uint32_t c = slice; c < count; c += 16) s += *reinterpret_cast<const f32x4*>(from + (size_t)c * stride);
    }
    slices[slice][quad] = s;
    __syncthreads();
    if (slice != 0 || e0 >= all) return;
    for (int i = 1; i < 16; ++i) s += slices[i][quad];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const size_t e = e0 + j;
        if (e < size) a.dw[(size_t)g * size + e] = s[j];
        else if (e < all && a.db) a.db[(size_t)g * a.out + (e - size)] = s[j];
    }
}

}  // namespace pcc_train
