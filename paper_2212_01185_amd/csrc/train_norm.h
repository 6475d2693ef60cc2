// Layer norm of rows, each with the weights of its group, and its backward pass.
//
//   h = (x - mean(x)) s,  s = 1 / sqrt(mean((x - mean(x))^2) + eps),  y = gamma h + beta
//   with u = gamma dy:  dx = s (u - mean(u) - h mean(u h)),  dgamma = sum over rows of dy h,  dbeta = sum of dy
//
// A row is read once: LANES lanes have it in registers, eight neighbours at a time, so the variance is that of the distances from the
// mean and not a difference of two large sums.
#pragma once

#include "train_rows.h"

namespace pcc_train {

struct Norm {
    const void* x;
    const void* dy;
    const float* gamma;     // or null: 1
    const float* beta;      // or null: 0
    const int64_t* off;     // or null: one group has all rows
    void* y;                // forward: y; backward: dx
    float* stats;           // of each row: mean, 1 / width
    float* dgamma;
    float* dbeta;
    float* partial;         // sums of one chunk, 2 * features values each
    size_t ldx, lddy, ldy;
    int64_t rows;
    int groups, features;
    float eps, inverse;     // 1 / features
    uint32_t shared_max;    // chunks of sums that the workspace has room for
    int log2;               // rows of a chunk: mult * 2^log2
    uint32_t mult;
};

__device__ __forceinline__ Chunk norm_chunk(const Norm& a, uint32_t b, bool empty) {
    if (a.off) return find_chunk(a.off, a.groups, a.rows, a.log2, a.mult, 1, b, empty);
    const int64_t size = (int64_t)a.mult << a.log2, lo = size * b, hi = lo + size < a.rows ? lo + size : a.rows;
    const uint32_t count = (uint32_t)((a.rows + size - 1) / size);
    if (b >= count && !(empty && b == 0)) return {-1, 0, 0, 0, 0, 0};
    return {0, lo, hi, b, count ? count : 1, 0};
}

// Threads of a workgroup, and rows that it has at a time.
constexpr int norm_threads(int lanes) { return lanes <= 64 ? 256 : lanes; }
constexpr int norm_teams(int lanes) { return norm_threads(lanes) / lanes; }

// Sums over a row's lanes, the same in all of them.  More than a wave meet in LDS; `turn` tells the place, of two, so that one barrier is enough.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float (*meet)[16], int turn) {
    if constexpr (LANES <= 64) {
        return lanes_sum<LANES>(v);
    } else {
        v = lanes_sum<64>(v);
        if ((threadIdx.x & 63) == 0) meet[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) s += meet[turn][w];
        return s;
    }
}

template <class X, class Y, int LANES, int N>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_kernel(Norm a) {
    constexpr int kTeams = norm_teams(LANES);
    __shared__ float meet[2][16];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const int n = (int)(ch.hi - ch.lo);
    const float* gamma = a.gamma ? a.gamma + (size_t)ch.group * a.features : nullptr;
    const float* beta = a.beta ? a.beta + (size_t)ch.group * a.features : nullptr;
    for (int r0 = 0; r0 < n; r0 += kTeams) {
        // a row behind the chunk's last is that one again
        const bool mine = r0 + team < n;
        const size_t row = (size_t)ch.lo + (mine ? r0 + team : n - 1);
        Eight<X> x[N];
        float sum = 0.0f, squares = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            x[i].load(a.x, row * a.ldx + f, a.features - f);
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[i].get(e);
        const float mean = row_sum<LANES>(sum, meet, 0) * a.inverse;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int left = a.features - 8 * (lane + LANES * i);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x[i].get(e) - mean;
                squares += e < left ? d * d : 0.0f;
            }
        }
        const float scale = 1.0f / sqrtf(row_sum<LANES>(squares, meet, 1) * a.inverse + a.eps);
        if (!mine) continue;
        if (a.stats && lane == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = scale;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            if (f >= a.features) continue;
            Eight<Fp32> w, b;
            if (gamma) w.load(gamma, f, a.features - f);
            if (beta) b.load(beta, f, a.features - f);
            Eight<Y> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = (x[i].get(e) - mean) * scale;
                y.set(e, __builtin_fmaf(gamma ? w.get(e) : 1.0f, h, beta ? b.get(e) : 0.0f));
            }
            y.store(a.y, row * a.ldy + f, a.features - f);
        }
    }
}

// dx of rows.
template <class X, class Y, int LANES, int N>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_dx_kernel(Norm a) {
    constexpr int kTeams = norm_teams(LANES);
    __shared__ float meet[4][16];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    const int n = (int)(ch.hi - ch.lo);
    const float* gamma = a.gamma ? a.gamma + (size_t)ch.group * a.features : nullptr;
    int turn = 0;
    for (int r0 = 0; r0 < n; r0 += kTeams, turn ^= 2) {
        const bool mine = r0 + team < n;
        const size_t row = (size_t)ch.lo + (mine ? r0 + team : n - 1);
        const float mean = a.stats[2 * row], scale = a.stats[2 * row + 1];
        Eight<X> x[N];
        Eight<Y> dy[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            x[i].load(a.x, row * a.ldx + f, a.features - f);
            dy[i].load(a.dy, row * a.lddy + f, a.features - f);
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            Eight<Fp32> w;
            if (gamma) w.load(gamma, f, a.features - f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = dy[i].get(e) * (gamma ? w.get(e) : 1.0f), h = (x[i].get(e) - mean) * scale;
                s1 += f + e < a.features ? u : 0.0f;
                s2 += f + e < a.features ? u * h : 0.0f;
            }
        }
        s1 = row_sum<LANES>(s1, meet, turn) * a.inverse;
        s2 = row_sum<LANES>(s2, meet, turn + 1) * a.inverse;
        if (!mine) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int f = 8 * (lane + LANES * i);
            if (f >= a.features) continue;
            Eight<Fp32> w;
            if (gamma) w.load(gamma, f, a.features - f);
            Eight<X> dx;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = dy[i].get(e) * (gamma ? w.get(e) : 1.0f), h = (x[i].get(e) - mean) * scale;
                dx.set(e, scale * (u - s1 - h * s2));
            }
            dx.store(a.y, row * a.ldy + f, a.features - f);
        }
    }
}

// Rows that do not fit the registers of a workgroup are read again for each sum: 1024 threads a row.
constexpr int kLongThreads = 1024;

template <class X, class Y>
__global__ __launch_bounds__(kLongThreads) void layer_norm_long_kernel(Norm a) {
    __shared__ float meet[2][16];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const float* gamma = a.gamma ? a.gamma + (size_t)ch.group * a.features : nullptr;
    const float* beta = a.beta ? a.beta + (size_t)ch.group * a.features : nullptr;
    for (int64_t row = ch.lo; row < ch.hi; ++row) {
        const size_t at = (size_t)row * a.ldx;
        float sum = 0.0f, squares = 0.0f;
        for (int f = 8 * threadIdx.x; f < a.features; f += 8 * kLongThreads) {
            Eight<X> x;
            x.load(a.x, at + f, a.features - f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x.get(e);
        }
        const float mean = row_sum<kLongThreads>(sum, meet, 0) * a.inverse;
        for (int f = 8 * threadIdx.x; f < a.features; f += 8 * kLongThreads) {
            Eight<X> x;
            x.load(a.x, at + f, a.features - f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x.get(e) - mean;
                squares += f + e < a.features ? d * d : 0.0f;
            }
        }
        const float scale = 1.0f / sqrtf(row_sum<kLongThreads>(squares, meet, 1) * a.inverse + a.eps);
        if (a.stats && threadIdx.x == 0) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = scale;
        }
        for (int f = 8 * threadIdx.x; f < a.features; f += 8 * kLongThreads) {
            Eight<X> x;
            Eight<Fp32> w, b;
            Eight<Y> y;
            x.load(a.x, at + f, a.features - f);
            if (gamma) w.load(gamma, f, a.features - f);
            if (beta) b.load(beta, f, a.features - f);
#pragma unroll
            for (int e = 0; e < 8; ++e) y.set(e, __builtin_fmaf(gamma ? w.get(e) : 1.0f, (x.get(e) - mean) * scale, beta ? b.get(e) : 0.0f));
            y.store(a.y, (size_t)row * a.ldy + f, a.features - f);
        }
    }
}

template <class X, class Y>
__global__ __launch_bounds__(kLongThreads) void layer_norm_long_dx_kernel(Norm a) {
    __shared__ float meet[4][16];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const float* gamma = a.gamma ? a.gamma + (size_t)ch.group * a.features : nullptr;
    int turn = 0;
    for (int64_t row = ch.lo; row < ch.hi; ++row, turn ^= 2) {
        const float mean = a.stats[2 * row], scale = a.stats[2 * row + 1];
        float s1 = 0.0f, s2 = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {
            for (int f = 8 * threadIdx.x; f < a.features; f += 8 * kLongThreads) {
                Eight<X> x, dx;
                Eight<Y> dy;
                Eight<Fp32> w;
                x.load(a.x, (size_t)row * a.ldx + f, a.features - f);
                dy.load(a.dy, (size_t)row * a.lddy + f, a.features - f);
                if (gamma) w.load(gamma, f, a.features - f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float u = dy.get(e) * (gamma ? w.get(e) : 1.0f), h = (x.get(e) - mean) * scale;
                    if (pass == 0) {
                        s1 += f + e < a.features ? u : 0.0f;
                        s2 += f + e < a.features ? u * h : 0.0f;
                    } else {
                        dx.set(e, scale * (u - s1 - h * s2));
                    }
                }
                if (pass == 1) dx.store(a.y, (size_t)row * a.ldy + f, a.features - f);
            }
            if (pass == 0) {
                s1 = row_sum<kLongThreads>(s1, meet, turn) * a.inverse;
                s2 = row_sum<kLongThreads>(s2, meet, turn + 1) * a.inverse;
            }
        }
    }
}

// Sums over the rows of a chunk: a thread has eight columns, 32 threads the rows in turn.
template <class X, class Y>
__global__ __launch_bounds__(256) void layer_norm_sums_kernel(Norm a) {
    __shared__ float slices[8][32][17];
    const Chunk ch = norm_chunk(a, blockIdx.x, true);
    if (ch.group < 0 || (ch.count > 1 && ch.shared >= a.shared_max)) return;
    const int n = (int)(ch.hi - ch.lo), slice = threadIdx.x >> 5;
    float* to = ch.count == 1 ? a.dgamma + (size_t)ch.group * a.features : a.partial + (size_t)ch.shared * 2 * a.features;
    float* to_beta = ch.count == 1 ? a.dbeta + (size_t)ch.group * a.features : to + a.features;
    for (int f0 = 256 * blockIdx.y; f0 < a.features; f0 += 256 * gridDim.y) {
        const int f = f0 + 8 * (threadIdx.x & 31);
        float dg[8] = {}, db[8] = {};
        if (f < a.features) {
            for (int r = slice; r < n; r += 8) {
                const size_t row = (size_t)ch.lo + r;
                const float mean = a.stats[2 * row], scale = a.stats[2 * row + 1];
                Eight<X> x;
                Eight<Y> dy;
                x.load(a.x, row * a.ldx + f, a.features - f);
                dy.load(a.dy, row * a.lddy + f, a.features - f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dg[e] += dy.get(e) * ((x.get(e) - mean) * scale);
                    db[e] += dy.get(e);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            slices[slice][threadIdx.x & 31][e] = dg[e];
            slices[slice][threadIdx.x & 31][8 + e] = db[e];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 512; i += 256) {
            const int column = i & 255, which = i >> 8;
            float s = 0.0f;
            for (int k = 0; k < 8; ++k) s += slices[k][column >> 3][8 * which + (column & 7)];
            if (f0 + column < a.features) (which ? to_beta : to)[f0 + column] = s;
        }
        __syncthreads();
    }
}

// Chunks' sums to those of their group, always in the same order.  A group of one chunk was written where it belongs.
__global__ __launch_bounds__(256) void layer_norm_join_kernel(Norm a) {
    __shared__ float slices[4][64];
    const int g = blockIdx.y, lane = threadIdx.x & 63;
    int64_t lo, hi;
    uint32_t count, first = 0;
    if (a.off) {
        count = uniform(group_chunks(a.off, g, a.groups, a.rows, a.log2, a.mult, true, lo, hi));
        if (count <= 1) return;
        if (a.groups > 64) {
            first = uniform(shared_place(lo, g, a.groups, a.rows, a.log2, a.mult));
        } else {
            const uint32_t n = group_chunks(a.off, lane, g, a.rows, a.log2, a.mult, true, lo, hi);
            first = wave_sum(n > 1 ? n : 0);
        }
    } else {
        const int64_t size = (int64_t)a.mult << a.log2;
        count = (uint32_t)((a.rows + size - 1) / size);
        if (count <= 1) return;
    }
    if (first + count > a.shared_max) return;
    const int all = 2 * a.features, slice = threadIdx.x >> 6;
    for (int e0 = 64 * blockIdx.x; e0 < all; e0 += 64 * gridDim.x) {
        const int e = e0 + lane;
        float s = 0.0f;
        if (e < all) {
            const float* from = a.partial + (size_t)first * all + e;
#pragma unroll 4
            for (uint32_t c = slice; c < count; c += 4) s += from[(size_t)c * all];
        }
        slices[slice][lane] = s;
        __syncthreads();
        if (slice == 0 && e < all) {
            s = slices[0][lane] + slices[1][lane] + slices[2][lane] + slices[3][lane];
            (e < a.features ? a.dgamma + (size_t)g * a.features + e : a.dbeta + (size_t)g * a.features + (e - a.features))[0] = s;
        }
        __syncthreads();
    }
}

}  // namespace pcc_train
