// Products of rows with few features, as the codec's layers have them: a group's weights fit a compute unit's LDS, rows are read
// once and written once, and memory sets the time (160 to 160: 640 bytes and 51,200 operations a row, 80 a byte, where the chip
// has 230 of the one for one of the other).
#pragma once

#include "train_grouped.h"

namespace pcc_train {

// ---------------------------------------------------------------------------
// Forward.  A workgroup of eight waves takes a chunk of one group's rows, a wave 32 of them at a time: rows are the product's
// n, read from memory as MFMA operands (a lane 16 bytes of one row; four lanes have 64 bytes of it), the next 32 while
// these are multiplied.  The weights are in LDS as operands.  Two blocks of 16 outputs are made together, their outputs
// dealt so that a lane gets eight neighbours: block b, row 4 g + i is output 32 pair + 8 g + 4 b + i.  Finished rows go through LDS where
// it has room, so that they leave in whole lines (160 to 160 on 393,216 rows, us: 72 without, 64 with: 3.9 TB/s, a large copy has
// 5.2; 786,432 rows 4.3 TB/s).  One workgroup of 512 threads a compute unit: with 256 threads, or with registers for four waves a
// SIMD, 79 to 87 us.  What is left is the start (the offsets, the weights: some 4 us) and reading 64 bytes of a row at a time;
// nothing is fetched or written twice, and the vector ALU is busy for 45 %, the matrix cores for 17 % of the time.
// ---------------------------------------------------------------------------
constexpr int kNarrowThreads = 512, kNarrowRowsWave = 32;

__host__ __device__ constexpr size_t narrow_forward_lds(int in, int out) {
    const size_t pairs = ((size_t)out + 31) / 32, kb = ((size_t)in + 31) / 32;
    return pairs * 2 * kb * 1024 + pairs * 32 * sizeof(float);
}
// A wave's outputs of 32 rows on their way to memory; a row's bytes, in whole pieces of 16 and one more.
__host__ __device__ constexpr int narrow_row_pieces(int features, int y32) { return (features * (y32 ? 4 : 2) + 15) / 16; }
__host__ __device__ constexpr size_t narrow_rows_lds(int features, int y32) { return (size_t)kNarrowRowsWave * (narrow_row_pieces(features, y32) + 1) * 16; }

// The row of a wave's piece, id / pieces, by a product: exact for all rows of up to 50 pieces (with 51, piece 1,325 would be the one before
// row 26's first).
constexpr int kMaxRowPieces = 50;
__host__ __device__ constexpr uint32_t pieces_inverse(int pieces) { return (65536 + pieces - 1) / pieces; }
__host__ __device__ constexpr int row_of_piece(int id, uint32_t inverse) { return (int)((uint32_t)id * inverse >> 16); }
constexpr bool rows_of_pieces_are_exact(int pieces) {
    for (int id = 0; id < kNarrowRowsWave * pieces; ++id)
        if (row_of_piece(id, pieces_inverse(pieces)) != id / pieces) return false;
    return pieces == 1 || rows_of_pieces_are_exact(pieces - 1);
}
static_assert(rows_of_pieces_are_exact(kMaxRowPieces), "rows of pieces");

// Rows in LDS (of one wave) to memory, 16 bytes a lane, neighbours next to each other.
__device__ __forceinline__ void store_rows(const uint8_t* lds, uint8_t* to, size_t ld_bytes, int rows, int row_bytes) {
    const int pieces = (row_bytes + 15) / 16, lane = threadIdx.x & 63;
    const uint32_t inverse = pieces_inverse(pieces);
    for (int id = lane; id < rows * pieces; id += 64) {
        const int r = row_of_piece(id, inverse), c = id - r * pieces, left = row_bytes - 16 * c;
        const uint8_t* from = lds + (r * (pieces + 1) + c) * 16;
        uint8_t* at = to + (size_t)r * ld_bytes + 16 * c;
        if (left >= 16) { u32x4 v = *reinterpret_cast<const u32x4*>(from);
            typedef u32x4 at_four __attribute__((aligned(4)));
            __builtin_nontemporal_store(v, reinterpret_cast<at_four*>(at));
        }
        else {
            int e = 0;
            if (left & 8) { __builtin_memcpy(at, from, 8); e = 8; }
            if (left & 4) { __builtin_memcpy(at + e, from + e, 4); e += 4; }
            if (left & 2) __builtin_memcpy(at + e, from + e, 2);
        }
    }
}

template <class T, int KB>
__global__ __launch_bounds__(kNarrowThreads) void grouped_narrow_forward_kernel(Grouped a) {
    extern __shared__ __align__(16) u16 lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quad = lane >> 4;
    const int threads = blockDim.x, step = kNarrowRowsWave * (threads / 64);
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, 1, blockIdx.x, false);
    if (ch.group < 0) return;
    const int pairs = (a.out + 31) / 32;
    float* bias = reinterpret_cast<float*>(lds + (size_t)pairs * 2 * KB * 512);
    uint8_t* mine = reinterpret_cast<uint8_t*>(bias + 32 * pairs) + wave * narrow_rows_lds(a.out, a.y32);
    const int row_bytes = a.out * (a.y32 ? 4 : 2), stride = (narrow_row_pieces(a.out, a.y32) + 1) * 16;
    const u16* x = a.x + (size_t)ch.lo * a.ldx;
    const int n = (int)(ch.hi - ch.lo);             // of a chunk: at most 2^27 rows

    // rows of this wave from r0 on, as operands; a row behind the chunk's last is that one again
    auto read = [&](int r0, u16x8 (&to)[2][KB]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int r = r0 + 16 * t + col;
            const u16* from = x + (size_t)(r < n ? r : n - 1) * a.ldx + 8 * quad;
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                // the last block may have fewer than four chunks; features are a multiple of eight
                if (k + 1 < KB || 32 * k + 8 * quad < a.in) __builtin_memcpy(&to[t][k], from + 32 * k, 16);
                else to[t][k] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            }
        }
    };
    u16x8 now[2][KB], next[2][KB];
    int r0 = kNarrowRowsWave * wave;
    if (r0 < n) read(r0, now);

    const u16* w = a.w + (size_t)ch.group * a.in * a.out;
    const int slots = pairs * 2 * KB * 64;
    for (int s0 = threadIdx.x; s0 < slots; s0 += 4 * threads) {
        u16x8 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {           // four loads at a time: each waits for memory or L2
            const int slot = s0 + u * threads, m = slot & 15, chunk = (slot >> 4) & 3, k = slot / 64 % KB, b = slot / 64 / KB;
            const int f = 32 * (b >> 1) + 8 * (m >> 2) + 4 * (b & 1) + (m & 3), c = 32 * k + 8 * chunk;
            v[u] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (slot < slots && f < a.out && c < a.in) __builtin_memcpy(&v[u], w + (size_t)f * a.in + c, 16);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (s0 + u * threads < slots) *reinterpret_cast<u16x8*>(lds + (s0 + u * threads) * 8) = v[u];
    }
    for (int f = threadIdx.x; f < 32 * pairs; f += threads)
        bias[f] = a.bias && f < a.out ? a.bias[(size_t)ch.group * a.out + f] : 0.0f;
    __syncthreads();

    for (; r0 < n; r0 += step) {
        if (r0 + step < n) read(r0 + step, next);
        for (int pair = 0; pair < pairs; ++pair) {
            f32x4 acc[2][2] = {};
            const u16* p = lds + (size_t)pair * 2 * KB * 512 + lane * 8;
#pragma unroll
            for (int k = 0; k < KB; ++k) {
                const u16x8 p0 = *reinterpret_cast<const u16x8*>(p + k * 512), p1 = *reinterpret_cast<const u16x8*>(p + (KB + k) * 512);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    acc[t][0] = T::mfma(p0, now[t][k], acc[t][0]);
                    acc[t][1] = T::mfma(p1, now[t][k], acc[t][1]);
                }
            }
            const int f = 32 * pair + 8 * quad;
            const f32x4 b0 = *reinterpret_cast<const f32x4*>(bias + f), b1 = *reinterpret_cast<const f32x4*>(bias + f + 4);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (!a.staged) {
                    const int r = r0 + 16 * t + col;
                    if (r < n && f < a.out) store_eight<T>(a, (size_t)(ch.lo + r) * a.ldy + f, acc[t][0] + b0, acc[t][1] + b1, a.out - f, a.act);
                    continue;
                }
                f32x4 v0 = acc[t][0] + b0, v1 = acc[t][1] + b1;
#pragma unroll
                for (int e = 0; e < 4; ++e) { v0[e] = activate(v0[e], a.act); v1[e] = activate(v1[e], a.act); }
                uint8_t* at = mine + (16 * t + col) * stride + f * (a.y32 ? 4 : 2);
                if (a.y32) {
                    if (f < a.out) *reinterpret_cast<f32x4*>(at) = v0;
                    if (f + 4 < a.out) *reinterpret_cast<f32x4*>(at + 16) = v1;
                } else if (f < a.out) {
                    u16x8 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) { o[e] = to16<T>(v0[e]); o[4 + e] = to16<T>(v1[e]); }
                    *reinterpret_cast<u16x8*>(at) = o;
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
        if (a.staged) store_rows(mine, static_cast<uint8_t*>(a.y) + (size_t)(ch.lo + r0) * a.ldy * (a.y32 ? 4 : 2), a.ldy * (a.y32 ? 4 : 2),
                   n - r0 < kNarrowRowsWave ? n - r0 : kNarrowRowsWave, row_bytes);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < KB; ++k) now[t][k] = next[t][k];
    }
}

// ---------------------------------------------------------------------------
// Backward, all of it in one pass over dz and x: every row of both is read once.  A workgroup of eight waves takes a chunk of
// one group's rows in steps of 64 (32 where LDS has no room for more); a step's rows of dz and x go to LDS by registers, the
// next step's on the way while this one's are multiplied (loads that go to LDS by themselves would be waited for before every
// ds_read_b64_tr_b16: the compiler cannot tell which of them it must see).  From there dz is read along for dx, and dz and x
// across for dw, whose sums stay in registers to the chunk's end (the waves have a part of dw each: halves of the inputs,
// quarters of the outputs).
// A row in LDS has its chunks of 8 values, zeros up to a multiple of four chunks, and two more of nothing: a distance of 2 modulo 4
// chunks puts the 32-byte pieces of eight rows, which ds_read_b64_tr_b16 reads together, into different banks.
// 160 to 160 on 393,216 rows: 99 us (3.8 TB/s), 5 of them for joining 256 chunks' sums; with loads straight to LDS 135 us, and as two passes
// of the tile kernel 348.  LDS is busy for 36 % of the time, matrix cores and vector ALU for 26 and 30; the rest is memory, and 24 us of start and end
// (a chunk's sums are 100 KB).
// ---------------------------------------------------------------------------
constexpr int kMaxLds = 160 * 1024;

// PAIRS, KBS: inputs, outputs in units of 32.
template <int PAIRS, int KBS>
struct NarrowBackward {
    static constexpr int kXChunks = 4 * PAIRS + 2, kZChunks = 4 * KBS + 2;      // of a row in LDS
    static constexpr size_t kWeights = (size_t)PAIRS * 2 * KBS * 1024;          // w^T as operands
    static constexpr size_t tiles(int rows) { return 2 * (size_t)rows * (kXChunks + kZChunks) * 16; }
    static constexpr int kRows = kWeights + tiles(64) <= kMaxLds ? 64 : 32;
    static constexpr size_t kLds = kWeights + tiles(kRows);
    static_assert(kLds <= kMaxLds, "LDS");
    static constexpr int kXLoads = (kRows * 4 * PAIRS + kNarrowThreads - 1) / kNarrowThreads;
    static constexpr int kZLoads = (kRows * 4 * KBS + kNarrowThreads - 1) / kNarrowThreads;
    static constexpr int kNB = (KBS + 1) / 2;       // blocks of 16 outputs of a wave
    static constexpr int kWRows = 32 * (int)(tiles(kRows) / ((size_t)32 * kXChunks * 16) < KBS ? tiles(kRows) / ((size_t)32 * kXChunks * 16) : KBS);
};

// A thread's chunks of `rows` rows of 32 * UNITS features (zeros where there is nothing), in registers between memory and LDS.
template <int UNITS, int LOADS>
struct RowPieces {
    u32x4 v[LOADS];
    __device__ void load(const u16* base, size_t ld, int features, int rows, int left) {
#pragma unroll
        for (int s = 0; s < LOADS; ++s) {
            const int slot = threadIdx.x + kNarrowThreads * s, r = slot / (4 * UNITS), c = slot % (4 * UNITS), there = features - 8 * c;
            u32x4 u = {0, 0, 0, 0};
            if (r < left && r < rows && there > 0) {
                const u16* from = base + (size_t)r * ld + 8 * c;
                if (there >= 8) __builtin_memcpy(&u, from, 16);
                else {                              // the chunk that the row's end cuts: features are even
                    const uint32_t* words = reinterpret_cast<const uint32_t*>(from);
                    u[0] = words[0];
                    if (there > 2) u[1] = words[1];
                    if (there > 4) u[2] = words[2];
                }
            }
            v[s] = u;
        }
    }
    __device__ void store(u16* lds, int rows) const {
#pragma unroll
        for (int s = 0; s < LOADS; ++s) {
            const int slot = threadIdx.x + kNarrowThreads * s, r = slot / (4 * UNITS), c = slot % (4 * UNITS);
            if (r < rows) *reinterpret_cast<u32x4*>(lds + (r * (4 * UNITS + 2) + c) * 8) = v[s];
        }
    }
};

__device__ __forceinline__ u16x8 read_across(const u16* at, int row_values) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const u16x4 a = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at));
    const u16x4 b = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * row_values)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <class T, int PAIRS, int KBS>
__global__ __launch_bounds__(kNarrowThreads) void grouped_narrow_backward_kernel(Grouped a) {
    using L = NarrowBackward<PAIRS, KBS>;
    constexpr int kRows = L::kRows, kXRow = L::kXChunks * 8, kZRow = L::kZChunks * 8, NB = L::kNB;
    extern __shared__ __align__(16) u16 lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, 1, blockIdx.x, true);
    if (ch.group < 0 || (ch.count > 1 && ch.shared >= a.shared_max)) return;    // (the second only with offsets that fall)
    const int n = (int)(ch.hi - ch.lo);
    const u16* dz = a.dz + (size_t)ch.lo * a.lddz;
    const u16* x = a.x + (size_t)ch.lo * a.ldx;
    u16* tiles = lds + L::kWeights / 2;
    RowPieces<KBS, L::kZLoads> z_next;
    RowPieces<PAIRS, L::kXLoads> x_next;
    z_next.load(dz, a.lddz, a.out, kRows, n);
    x_next.load(x, a.ldx, a.in, kRows, n);

    // a lane's place when 32 rows are read across: row 8 quad + (lane % 16) / 4 (and four below it), column 4 (lane % 4) of 16
    const int across_row = 8 * quad + (col >> 2), across_col = 4 * (lane & 3);
    if (a.y) {
        // w^T as operands: inputs are dealt to two blocks of a pair as the forward kernel deals its outputs
        const u16* w = a.w + (size_t)ch.group * a.in * a.out;
        for (int o0 = 0; o0 < 32 * KBS; o0 += L::kWRows) {
            for (int i = threadIdx.x; i < L::kWRows * 4 * PAIRS; i += kNarrowThreads) {
                const int o = i / (4 * PAIRS), c = i % (4 * PAIRS);
                u32x4 v = {0, 0, 0, 0};
                if (o0 + o < a.out && 8 * c < a.in) __builtin_memcpy(&v, w + (size_t)(o0 + o) * a.in + 8 * c, 16);
                *reinterpret_cast<u32x4*>(tiles + o * kXRow + 8 * c) = v;
            }
            __syncthreads();
            for (int i = wave; i < L::kWRows / 32 * 2 * PAIRS; i += 8) {
                const int k = i / (2 * PAIRS), b = i % (2 * PAIRS);
                if (o0 / 32 + k < KBS) {
                    const u16x8 v = read_across(tiles + (32 * k + across_row) * kXRow + 32 * (b >> 1) + 2 * across_col + 4 * (b & 1), kXRow);
                    *reinterpret_cast<u16x8*>(lds + ((b * KBS + o0 / 32 + k) * 64 + lane) * 8) = v;
                }
            }
            __syncthreads();
        }
    }
    z_next.store(tiles, kRows);
    x_next.store(tiles + kRows * kZRow, kRows);

    // blocks of 16 of dw; the last of a wave's may be another's as well (and is not stored)
    const int mb0 = (wave & 1) * PAIRS, nb0 = (wave >> 1) * NB;
    f32x4 acc[PAIRS][NB] = {}, sums[NB] = {};
    u16x8 ones;
    for (int j = 0; j < 8; ++j) ones[j] = T::kOne;
    const bool with_db = a.db && (wave & 1) == 0;
    constexpr int kRowTiles = kRows / 16, kPairStep = 8 / kRowTiles;
    const int my_row = 16 * (wave % kRowTiles) + col, pair0 = wave / kRowTiles;

    int now = 0;
    for (int r0 = 0; r0 < n; r0 += kRows, now ^= 1) {
        __syncthreads();
        const u16* zt = tiles + now * kRows * (kZRow + kXRow);
        const u16* xt = zt + kRows * kZRow;
        const bool more = r0 + kRows < n;
        if (more) {
            z_next.load(dz + (size_t)(r0 + kRows) * a.lddz, a.lddz, a.out, kRows, n - r0 - kRows);
            x_next.load(x + (size_t)(r0 + kRows) * a.ldx, a.ldx, a.in, kRows, n - r0 - kRows);
        }
        if (a.y) {
            u16x8 q[KBS];
#pragma unroll
            for (int k = 0; k < KBS; ++k) q[k] = *reinterpret_cast<const u16x8*>(zt + my_row * kZRow + 32 * k + 8 * quad);
#pragma unroll
            for (int j = 0; j < (PAIRS + kPairStep - 1) / kPairStep; ++j) {
                const int pair = pair0 + j * kPairStep;
                if (pair >= PAIRS) break;
                f32x4 d0 = {}, d1 = {};
                const u16* p = lds + (size_t)pair * 2 * KBS * 512 + lane * 8;
#pragma unroll
                for (int k = 0; k < KBS; ++k) {
                    d0 = T::mfma(*reinterpret_cast<const u16x8*>(p + k * 512), q[k], d0);
                    d1 = T::mfma(*reinterpret_cast<const u16x8*>(p + (KBS + k) * 512), q[k], d1);
                }
                // the products' results are complete on both sides of the branch: eight wait states, which the compiler counts on its own
                // in straight-line code only
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_nop 7");
                __builtin_amdgcn_sched_barrier(0);
                const int f = 32 * pair + 8 * quad;
                if (a.act != PCC_ACT_NONE) {
                    const u16x8 s = *reinterpret_cast<const u16x8*>(xt + my_row * kXRow + f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        d0[e] = times_derivative(d0[e], from16<T>(s[e]), a.act);
                        d1[e] = times_derivative(d1[e], from16<T>(s[4 + e]), a.act);
                    }
                }
                if (r0 + my_row < n && f < a.in) {
                    u16x8 o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) { o[e] = to16<T>(d0[e]); o[4 + e] = to16<T>(d1[e]); }
                    u16* to = static_cast<u16*>(a.y) + (size_t)(ch.lo + r0 + my_row) * a.ldy + f;
                    __builtin_memcpy(to, &o, 16);       // inputs are a multiple of eight, in rows that begin at even elements
                }
            }
        }
#pragma unroll
        for (int kk = 0; kk < kRows / 32; ++kk) {
            u16x8 q[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int nb = nb0 + j < 2 * KBS ? nb0 + j : 2 * KBS - 1;
                q[j] = read_across(zt + (32 * kk + across_row) * kZRow + 16 * nb + across_col, kZRow);
            }
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                const u16x8 p = read_across(xt + (32 * kk + across_row) * kXRow + 16 * (mb0 + i) + across_col, kXRow);
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = T::mfma(p, q[j], acc[i][j]);
            }
            if (with_db)
#pragma unroll
                for (int j = 0; j < NB; ++j) sums[j] = T::mfma(ones, q[j], sums[j]);
        }
        if (more) {
            u16* to = tiles + (now ^ 1) * kRows * (kZRow + kXRow);
            z_next.store(to, kRows);
            x_next.store(to + kRows * kZRow, kRows);
        }
    }

    const size_t size = (size_t)a.in * a.out;
    float* dw = ch.count == 1 ? a.dw + (size_t)ch.group * size : a.partial + (size_t)ch.shared * partial_values(a.in, a.out);
    float* db = ch.count == 1 ? a.db + (a.db ? (size_t)ch.group * a.out : 0) : dw + size;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int o = 16 * (nb0 + j) + col;
        if (o >= a.out) continue;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const int f = 16 * (mb0 + i) + 4 * quad;
            if (f < a.in) store_four(dw + (size_t)o * a.in + f, acc[i][j], 4, a.wide_dw);
        }
        if (with_db && quad == 0) db[o] = sums[j][0];
    }
}

}  // namespace pcc_train
