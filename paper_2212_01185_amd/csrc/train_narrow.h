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
// dealt so that a lane gets eight neighbours: block b, row 4 g + i is output 32 pair + 8 g + 4 b + i.
// ---------------------------------------------------------------------------
constexpr int kNarrowThreads = 512, kNarrowRowsWave = 32;

__host__ __device__ constexpr size_t narrow_forward_lds(int in, int out) {
    const size_t pairs = ((size_t)out + 31) / 32, kb = ((size_t)in + 31) / 32;
    return pairs * 2 * kb * 1024 + pairs * 32 * sizeof(float);
}
// A wave's outputs of 32 rows on their way to memory; a row's bytes, in whole pieces of 16 and one more.
__host__ __device__ constexpr int narrow_row_pieces(int features, int y32) { return (features * (y32 ? 4 : 2) + 15) / 16; }
__host__ __device__ constexpr size_t narrow_rows_lds(int features, int y32) { return (size_t)kNarrowRowsWave * (narrow_row_pieces(features, y32) + 1) * 16; }

// Rows in LDS (of one wave) to memory, 16 bytes a lane, neighbours next to each other.
__device__ __forceinline__ void store_rows(const uint8_t* lds, uint8_t* to, size_t ld_bytes, int rows, int row_bytes) {
    const int pieces = (row_bytes + 15) / 16, lane = threadIdx.x & 63;
    const uint32_t inverse = (65536 + pieces - 1) / pieces;         // exact for pieces of up to 2,048 numbers
    for (int id = lane; id < rows * pieces; id += 64) {
        const int r = (int)((uint32_t)id * inverse >> 16), c = id - r * pieces, left = row_bytes - 16 * c;
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
// one group's rows in steps of 64 (32 where LDS has no room for more); a step's rows of dz and x go to LDS, the next step's on
// the way while this one's are multiplied.  From there dz is read along for dx, and dz and x across for dw, whose sums stay in
// registers to the chunk's end (the waves have a part of dw each: halves of the inputs, quarters of the outputs).
// A row in LDS has its chunks of 8 values, zeros up to a multiple of four chunks, and two more of nothing: a distance of 2 modulo 4
// chunks puts the 32-byte pieces of eight rows, which ds_read_b64_tr_b16 reads together, into different banks.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr int narrow_chunks(int features) { return (features + 31) / 32 * 4 + 2; }
__host__ __device__ constexpr size_t narrow_backward_lds(int in, int out, int rows, bool dx) {
    const size_t weights = dx ? ((size_t)in + 31) / 32 * 2 * (((size_t)out + 31) / 32) * 1024 : 0;
    return weights + 2 * (size_t)rows * (narrow_chunks(in) + narrow_chunks(out)) * 16;
}

// A thread's part in bringing a step's rows to LDS.
struct NarrowSource {
    static constexpr uint32_t kSkip = 0xFFFFFFFFu, kNone = 0x7FFFFF00u;
    uint32_t offset[4];
    const u16* base;
    size_t ld;
    int chunks, cut;        // chunks of a row in LDS; values of the chunk that the row's end cuts
    int features;

    __device__ void init(const u16* b, size_t stride, int n_features, int rows) {
        base = b;
        ld = stride;
        features = n_features;
        chunks = narrow_chunks(n_features);
        cut = n_features % 8;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int slot = threadIdx.x + kNarrowThreads * s, r = slot / chunks, c = slot - r * chunks;
            offset[s] = r < rows && 8 * c + 8 <= n_features ? (uint32_t)(((size_t)r * ld + 8 * c) * 2) : kSkip;
        }
    }
    // Zeros in what no load writes: the chunks behind a row's last.
    __device__ void clear(u16* lds, int rows) const {
        const int first = features / 8, last = (features + 31) / 32 * 4;
        for (int i = threadIdx.x; i < rows * (last - first); i += kNarrowThreads) {
            const int r = i / (last - first), c = first + i - r * (last - first);
            *reinterpret_cast<u16x8*>(lds + (r * chunks + c) * 8) = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
        }
    }
    // Rows r0 .. of the chunk, `left` of them there; zeros for the others.
    __device__ void stage(u16* lds, int64_t r0, int left) const {
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (size_t)r0 * ld), 0, (int)kNone, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            if (offset[s] == kSkip) continue;
            const bool there = (int)((threadIdx.x + kNarrowThreads * s) / (uint32_t)chunks) < left;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)(lds + (64 * wave + kNarrowThreads * s) * 8), 16, there ? offset[s] : kNone, 0, 0, 0);
        }
    }
    // The chunk that the row's end cuts, of row threadIdx.x.
    __device__ u16x8 cut_chunk(int64_t r0, int left) const {
        u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        if ((int)threadIdx.x < left) {
            const u16* from = base + (size_t)(r0 + threadIdx.x) * ld + features - cut;
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < cut) v[j] = from[j];
        }
        return v;
    }
};

// Operand of 16 indices (chunk columns 2 i, 2 i + 1) and 32 rows from 32 kk on, read across.
__device__ __forceinline__ u16x8 across(const u16* lds, int chunks, int i, int kk, int lane) {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int r = 32 * kk + 8 * (lane >> 4) + ((lane & 15) >> 2), at = (r * chunks + 2 * i + ((lane & 3) >> 1)) * 8 + 4 * (lane & 1);
    const u16x4 a = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at)));
    const u16x4 b = __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at + 4 * chunks * 8)));
    u16x8 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = a[j]; v[j + 4] = b[j]; }
    return v;
}

// MB, NB: blocks of 16 inputs, outputs that a wave may have of dw.
template <class T, int MB, int NB>
__global__ __launch_bounds__(kNarrowThreads) void grouped_narrow_backward_kernel(Grouped a) {
    extern __shared__ __align__(16) u16 lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const Chunk ch = find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, 1, blockIdx.x, true);
    if (ch.group < 0) return;
    const int n = (int)(ch.hi - ch.lo), rows = a.step_rows;
    const int pairs = (a.in + 31) / 32, kbs = (a.out + 31) / 32;
    u16* tiles = lds + (a.y ? (size_t)pairs * 2 * kbs * 512 : 0);
    const int z_size = rows * narrow_chunks(a.out) * 8, x_size = rows * narrow_chunks(a.in) * 8;
    NarrowSource z, x;
    z.init(a.dz + (size_t)ch.lo * a.lddz, a.lddz, a.out, rows);
    x.init(a.x + (size_t)ch.lo * a.ldx, a.ldx, a.in, rows);
    auto z_tile = [&](int b) { return tiles + b * (z_size + x_size); };
    auto x_tile = [&](int b) { return tiles + b * (z_size + x_size) + z_size; };
    const bool cuts = z.cut != 0 && (int)threadIdx.x < rows;
    const int cut_at = ((int)threadIdx.x * z.chunks + a.out / 8) * 8;
    if (n > 0) {
        z.stage(z_tile(0), 0, n);
        x.stage(x_tile(0), 0, n);
    }
    for (int b = 0; b < 2; ++b) { z.clear(z_tile(b), rows); x.clear(x_tile(b), rows); }
    __syncthreads();
    if (cuts) *reinterpret_cast<u16x8*>(z_tile(0) + cut_at) = z.cut_chunk(0, n);

    if (a.y) {
        // w^T as operands: inputs are dealt to two blocks of a pair as the forward kernel deals its outputs
        const u16* w = a.w + (size_t)ch.group * a.in * a.out;
        for (int slot = threadIdx.x; slot < pairs * 2 * kbs * 64; slot += kNarrowThreads) {
            const int m = slot & 15, q = (slot >> 4) & 3, k = slot / 64 % kbs, b = slot / 64 / kbs;
            const int f = 32 * (b >> 1) + 8 * (m >> 2) + 4 * (b & 1) + (m & 3), o = 32 * k + 8 * q;
            u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (f < a.in && o + j < a.out) v[j] = w[(size_t)(o + j) * a.in + f];
            *reinterpret_cast<u16x8*>(lds + slot * 8) = v;
        }
    }

    const int m_blocks = (a.in + 15) / 16, n_blocks = (a.out + 15) / 16, m_each = (m_blocks + 1) / 2, n_each = (n_blocks + 3) / 4;
    const int mb0 = (wave & 1) * m_each, nb0 = (wave >> 1) * n_each;
    const int mbs = m_blocks - mb0 < m_each ? m_blocks - mb0 : m_each, nbs = n_blocks - nb0 < n_each ? n_blocks - nb0 : n_each;
    f32x4 acc[MB][NB] = {}, sums[NB] = {};
    u16x8 ones;
    for (int j = 0; j < 8; ++j) ones[j] = T::kOne;
    const bool with_db = a.db && (wave & 1) == 0;
    const int row_tiles = rows / 16, my_tile = wave % row_tiles, pair0 = wave / row_tiles, pair_step = 8 / row_tiles;

    int now = 0;
    for (int r0 = 0; r0 < n; r0 += rows, now ^= 1) {
        __builtin_amdgcn_s_waitcnt(0);          // this step's rows are in LDS, and the chunks that a thread wrote
        __syncthreads();
        const u16* zt = z_tile(now);
        const u16* xt = x_tile(now);
        u16x8 cut = {0, 0, 0, 0, 0, 0, 0, 0};
        const bool more = r0 + rows < n;
        if (more) {
            z.stage(z_tile(now ^ 1), r0 + rows, n - r0 - rows);
            x.stage(x_tile(now ^ 1), r0 + rows, n - r0 - rows);
            if (cuts) cut = z.cut_chunk(r0 + rows, n - r0 - rows);
        }
        if (a.y) {
            const int r = 16 * my_tile + col;
            u16x8 q[2 * NB];
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k)
                if (k < kbs) q[k] = *reinterpret_cast<const u16x8*>(zt + (r * z.chunks + 4 * k + quad) * 8);
            for (int pair = pair0; pair < pairs; pair += pair_step) {
                f32x4 d0 = {}, d1 = {};
                const u16* p = lds + (size_t)pair * 2 * kbs * 512 + lane * 8;
#pragma unroll
                for (int k = 0; k < 2 * NB; ++k) {
                    if (k >= kbs) continue;
                    d0 = T::mfma(*reinterpret_cast<const u16x8*>(p + k * 512), q[k], d0);
                    d1 = T::mfma(*reinterpret_cast<const u16x8*>(p + (kbs + k) * 512), q[k], d1);
                }
                const int f = 32 * pair + 8 * quad;
                if (a.act != PCC_ACT_NONE) {
                    const u16x8 s = *reinterpret_cast<const u16x8*>(xt + (r * x.chunks + 4 * pair + quad) * 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        d0[e] = times_derivative(d0[e], from16<T>(s[e]), a.act);
                        d1[e] = times_derivative(d1[e], from16<T>(s[4 + e]), a.act);
                    }
                }
                if (r0 + r < n && f < a.in) store_eight<T>(a, (size_t)(ch.lo + r0 + r) * a.ldy + f, d0, d1, 8, PCC_ACT_NONE);
            }
        }
        for (int kk = 0; kk < rows / 32; ++kk) {
            u16x8 q[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j)
                if (j < nbs) q[j] = across(zt, z.chunks, nb0 + j, kk, lane);
#pragma unroll
            for (int i = 0; i < MB; ++i) {
                if (i >= mbs) continue;
                const u16x8 p = across(xt, x.chunks, mb0 + i, kk, lane);
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (j < nbs) acc[i][j] = T::mfma(p, q[j], acc[i][j]);
            }
            if (with_db)
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (j < nbs) sums[j] = T::mfma(ones, q[j], sums[j]);
        }
        if (more && cuts) *reinterpret_cast<u16x8*>(z_tile(now ^ 1) + cut_at) = cut;
    }

    const size_t size = (size_t)a.in * a.out;
    float* dw = ch.count == 1 ? a.dw + (size_t)ch.group * size : a.partial + (size_t)ch.id * (size + a.out);
    float* db = ch.count == 1 ? a.db + (a.db ? (size_t)ch.group * a.out : 0) : dw + size;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int o = 16 * (nb0 + j) + col;
        if (j >= nbs || o >= a.out) continue;
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int f = 16 * (mb0 + i) + 4 * quad;
            if (i < mbs && f < a.in) store_four(dw + (size_t)o * a.in + f, acc[i][j], 4, a.wide_dw);
        }
        if (with_db && quad == 0) db[o] = sums[j][0];
    }
}

}  // namespace pcc_train
