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
    uint32_t shared_max;    // chunks of sums that the workspace has room for
    int log2;           // rows of a chunk: mult * 2^log2
    uint32_t mult;
    int y32;            // y is fp32
    int staged;         // forward, narrow: outputs go through LDS
    int wide_out, wide_x, wide_dw;  // four values of a row of the result, of x, of dw can be stored, read in one piece
    uint32_t tiles_m, tiles_n;
};

constexpr int kTileK = 64;
__host__ __device__ constexpr int tile_threads(int tile) { return 2 * tile; }

// An operand's tile in LDS, TILE (128, 256) indices and 64 k.  Chunks of 8 values; chunk c of row r stands at slot c ^ swizzle(r) of the row, so that the
// rows that are read together lie in different banks.
//   along: rows are the operand's indices, 64 k each (8 chunks)
//   across: rows are the 64 k, TILE indices each (16 or 32 chunks)
template <bool ACROSS, int TILE>
struct TileLds {
    static constexpr int kChunks = ACROSS ? TILE / 8 : 8;
    __device__ static int at(int r, int c) { return (r * kChunks + (c ^ (ACROSS ? (2 * (r & 7)) : (r & 7)))) * 8; }
    // The MFMA operand of indices 16 i .. +15, k 32 kk .. +31.
    __device__ static u16x8 operand(const u16* lds, int i, int kk, int lane) {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const u16x8*>(lds + at(16 * i + (lane & 15), 4 * kk + (lane >> 4)));
        } else {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const int r = 32 * kk + 8 * (lane >> 4) + ((lane & 15) >> 2), c = 2 * i + ((lane & 3) >> 1), e = 4 * (lane & 1);
            const u16x4 a = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r, c) + e)));
            const u16x4 b = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r + 4, c) + e)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

typedef __attribute__((address_space(3))) void lds_void;

// An operand in memory, and a workgroup's way through it in steps of 64 k.  Where rows begin at even elements (WIDE), chunks go 16
// bytes a lane: by themselves, without a register, if all operands are read along (the compiler waits for all such loads
// before a ds_read_b64_tr_b16, of which it cannot tell what it must see), else by registers.  A chunk that is cut by the end of its row is
// read value by value, and what lies beyond the operand is zero (a lane's offset beyond the buffer's end loads zeros).  Rows
// at odd elements take the way by registers, with loads that may begin anywhere.
template <bool ACROSS, int TILE>
struct Source {
    static constexpr int kThreads = tile_threads(TILE);
    const u16* base;            // index i0, k 0
    size_t ld;
    int64_t ni, nk;             // indices from i0 on, all k
    uint32_t offset[4];         // bytes of this lane's chunks from base + the step
    u32x4 held[4];              // chunks on their way by registers
    static constexpr uint32_t kNone = 0xFFFFFF00u;      // beyond the buffer (rows are at most 2^22 values, a tile has 256)

    __device__ void init(const u16* b, size_t stride, int64_t i0, int64_t n_index, int64_t n_k) {
        const u16* from = b + (ACROSS ? (size_t)i0 : (size_t)i0 * stride);
        base = reinterpret_cast<const u16*>(uniform64(reinterpret_cast<int64_t>(from)));
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
        const int slot = threadIdx.x + kThreads * s;
        r = slot / TileLds<ACROSS, TILE>::kChunks;
        c = (slot % TileLds<ACROSS, TILE>::kChunks) ^ (ACROSS ? 2 * (r & 7) : (r & 7));
    }
    // Values of a chunk that are there, at k0.
    __device__ int values(int r, int c, int64_t k0) const {
        const int64_t n = ACROSS ? (k0 + r < nk ? ni - 8 * c : 0) : (r < ni ? nk - k0 - 8 * c : 0);
        return n < 0 ? 0 : n > 8 ? 8 : (int)n;
    }
    __device__ u32x4 one_by_one(int r, int c, int64_t k0, int n) const {
        const u16* from = base + (ACROSS ? (size_t)(k0 + r) * ld + 8 * c : (size_t)r * ld + (size_t)k0 + 8 * c);
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if (n == 8) {           // a whole chunk, at any address: one load (buffers want multiples of four)
            __builtin_memcpy(&v, from, 16);
            return __builtin_bit_cast(u32x4, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) v[j] = from[j];
        return __builtin_bit_cast(u32x4, v);
    }
    __device__ __amdgpu_buffer_rsrc_t buffer(int64_t k0) const {
        return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (ACROSS ? (size_t)k0 * ld : (size_t)k0)), 0, (int)kNone, 0x00020000);
    }
    // All chunks of the step are there, or not at all for every k.
    __device__ bool whole(int64_t k0) const { return k0 + kTileK <= nk && (!ACROSS || ni % 8 == 0 || ni >= TILE); }

    // Straight to LDS.
    __device__ void stage(u16* lds, int64_t k0) const {
        const __amdgpu_buffer_rsrc_t from = buffer(k0);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const bool all = whole(k0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            lds_void* to = (lds_void*)(lds + (64 * wave + kThreads * s) * 8);
            if (all) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to, 16, offset[s], 0, 0, 0);
            } else {
                int r, c;
                place(s, r, c);
                const int n = values(r, c, k0);
                if (n == 0 || n == 8) __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to, 16, n ? offset[s] : kNone, 0, 0, 0);
                else *reinterpret_cast<u32x4*>(lds + (threadIdx.x + kThreads * s) * 8) = one_by_one(r, c, k0, n);
            }
        }
    }
    // To registers, and from there to LDS.
    template <bool WIDE>
    __device__ void fetch(int64_t k0) {
        const __amdgpu_buffer_rsrc_t from = buffer(k0);
        if (WIDE && whole(k0)) {
#pragma unroll
            for (int s = 0; s < 4; ++s) held[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, offset[s], 0, 0));
            return;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            int r, c;
            place(s, r, c);
            const int n = values(r, c, k0);
            if (WIDE && (n == 0 || n == 8)) held[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, n ? offset[s] : kNone, 0, 0));
            else held[s] = one_by_one(r, c, k0, n);
        }
    }
    __device__ void put(u16* lds) const {
#pragma unroll
        for (int s = 0; s < 4; ++s) *reinterpret_cast<u32x4*>(lds + (threadIdx.x + kThreads * s) * 8) = held[s];
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

// Rates: forward, four groups of 2,048 rows, 2048 to 2048, 71 us (970 TFLOP/s; a large library product of this card has 1,176) with tiles of 256;
// sixteen of 512 rows, 1024 to 4096, 131 us (525), where a group's last tile is half empty and 656 tiles take three turns of 256 compute units.
// dx and dw, sixteen of 512 rows, 1024 to 2048, 97 and 84 us (350 and 410): tiles of 256 would spill (their rows pass through registers).
// TILE x TILE results of a workgroup: 128 by four waves with 64 x 64 each, 256 by eight with 128 x 64.  Two tiles in LDS for each
// operand: the next step's is filled while this one's is multiplied.
template <class T, int MODE, bool WIDE, int TILE>
__global__ __launch_bounds__(tile_threads(TILE), 2) void grouped_tile_kernel(Grouped a) {
    constexpr bool kPAcross = MODE != kForward, kQAcross = MODE == kWeights;
    constexpr int kTile = TILE, MI = TILE / 32;
    using P = TileLds<kPAcross, TILE>;
    using Q = TileLds<kQAcross, TILE>;
    extern __shared__ __align__(16) u16 lds_all[];
    auto lds = [&](int buffer, int operand) { return lds_all + (2 * buffer + operand) * TILE * kTileK; };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
    const uint32_t tiles = a.tiles_m * (MODE == kWeights ? a.tiles_n : 1);
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, tiles, blockIdx.x, MODE == kWeights);
    if (ch.group < 0 || (MODE == kWeights && ch.count > 1 && ch.shared >= a.shared_max)) return;     // (the second only with offsets that fall)
    const int64_t m0 = (int64_t)(ch.part % a.tiles_m) * kTile, n0 = MODE == kWeights ? (int64_t)(ch.part / a.tiles_m) * kTile : 0;
    const int64_t n_rows = ch.hi - ch.lo;
    const u16* w = a.w ? a.w + (size_t)ch.group * a.in * a.out : nullptr;
    const int64_t np = MODE == kForward ? a.out : a.in, nq = MODE == kWeights ? a.out : n_rows;
    const int64_t nk = MODE == kForward ? a.in : MODE == kBackward ? a.out : n_rows;
    Source<kPAcross, TILE> p;
    Source<kQAcross, TILE> q;
    p.init(MODE == kWeights ? a.x + (size_t)ch.lo * a.ldx : w, MODE == kWeights ? a.ldx : (size_t)a.in, m0, np, nk);
    if (MODE == kForward) q.init(a.x + (size_t)ch.lo * a.ldx, a.ldx, n0, nq, nk);
    else q.init(a.dz + (size_t)ch.lo * a.lddz, a.lddz, n0, nq, nk);

    f32x4 acc[MI][4] = {}, sums[4] = {};
    const bool with_db = MODE == kWeights && a.db && m0 == 0 && wm == 0;
    u16x8 ones;
    for (int j = 0; j < 8; ++j) ones[j] = T::kOne;
    constexpr bool kStraight = WIDE && MODE == kForward;
    if (nk > 0) {
        if constexpr (kStraight) {
            p.stage(lds(0, 0), 0);
            q.stage(lds(0, 1), 0);
        } else {
            p.template fetch<WIDE>(0);
            q.template fetch<WIDE>(0);
            p.put(lds(0, 0));
            q.put(lds(0, 1));
        }
    }
    int now = 0;
    for (int64_t k0 = 0; k0 < nk; k0 += kTileK, now ^= 1) {
        if (kStraight) __builtin_amdgcn_s_waitcnt(0);       // the barrier alone does not wait for loads that go to LDS
        __syncthreads();
        const bool more = k0 + kTileK < nk;
        if (more) {
            if constexpr (kStraight) {
                p.stage(lds(now ^ 1, 0), k0 + kTileK);
                q.stage(lds(now ^ 1, 1), k0 + kTileK);
            } else {
                p.template fetch<WIDE>(k0 + kTileK);
                q.template fetch<WIDE>(k0 + kTileK);
            }
        }
        // Groups of four products that share P's block i of half kk.  P's blocks are read two groups ahead and Q's of the second half
        // during the first, each between two groups: read where they are needed, every group would wait for LDS.
        const u16* tp = lds(now, 0);
        const u16* tq = lds(now, 1);
        u16x8 fq[2][4], fp[2 * MI];
        auto read_q = [&](int kk, int j) { fq[kk][j] = Q::operand(tq, 4 * wn + j, kk, lane); };
        auto read_p = [&](int g) { fp[g] = P::operand(tp, MI * wm + g % MI, g / MI, lane); };
#pragma unroll
        for (int j = 0; j < 4; ++j) read_q(0, j);
        read_p(0);
        read_p(1);
        constexpr int kP = kPAcross ? 2 : 1, kQ = kQAcross ? 2 : 1;     // LDS instructions of an operand
        __builtin_amdgcn_sched_group_barrier(0x100, 4 * kQ + 2 * kP, 0);
#pragma unroll
        for (int g = 0; g < 2 * MI; ++g) {
            const int kk = g / MI, i = g % MI;
            if (g + 2 < 2 * MI) {
                read_p(g + 2);
                __builtin_amdgcn_sched_group_barrier(0x100, kP, 0);
            }
            if (kk == 0 && i < 4) {
                read_q(1, i);
                __builtin_amdgcn_sched_group_barrier(0x100, kQ, 0);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = T::mfma(fp[g], fq[kk][j], acc[i][j]);
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        }
        if (with_db)
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[j] = T::mfma(ones, fq[1][j], T::mfma(ones, fq[0][j], sums[j]));
        if (!kStraight && more) {
            p.put(lds(now ^ 1, 0));
            q.put(lds(now ^ 1, 1));
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
            dw = a.partial + (size_t)ch.shared * partial_values(a.in, a.out);
            db = dw + size;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + 64 * wn + 16 * j + (lane & 15);
        if (n >= nq) continue;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int64_t m = m0 + 16 * MI * wm + 16 * i + 4 * (lane >> 4);
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
    int64_t lo, hi;
    const uint32_t count = uniform(group_chunks(a.off, g, a.groups, a.rows, a.log2, a.mult, true, lo, hi));
    if (count <= 1) return;
    uint32_t first;
    if (a.groups > 64) {
        first = uniform(shared_place(lo, g, a.groups, a.rows, a.log2, a.mult));
    } else {
        const uint32_t n = group_chunks(a.off, lane, g, a.rows, a.log2, a.mult, true, lo, hi);
        first = wave_sum(n > 1 ? n : 0);
    }
    if (first + count > a.shared_max) return;
    const size_t size = (size_t)a.in * a.out, all = size + a.out, stride = partial_values(a.in, a.out);
    const int quad = threadIdx.x & 15, slice = threadIdx.x >> 4;
    for (size_t e0 = (size_t)blockIdx.x * 64 + 4 * quad; e0 - 4 * quad < all; e0 += (size_t)gridDim.x * 64) {
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        if (e0 < all) {
            const float* from = a.partial + (size_t)first * stride + e0;
#pragma unroll 4
            for (uint32_t c = slice; c < count; c += 16) s += *reinterpret_cast<const f32x4*>(from + (size_t)c * stride);
        }
        slices[slice][quad] = s;
        __syncthreads();
        if (slice == 0 && e0 < all) {
            for (int i = 1; i < 16; ++i) s += slices[i][quad];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const size_t e = e0 + j;
                if (e < size) a.dw[(size_t)g * size + e] = s[j];
                else if (e < all && a.db) a.db[(size_t)g * a.out + (e - size)] = s[j];
            }
        }
        __syncthreads();
    }
}

}  // namespace pcc_train
