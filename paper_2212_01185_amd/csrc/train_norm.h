// Layer norm of rows, each with the weights of its group, and its backward pass.
//
//   h = (x - mean(x)) s,  s = 1 / sqrt(mean((x - mean(x))^2) + eps),  y = gamma h + beta
//   with u = gamma dy:  dx = s (u - mean(u) - h mean(u h)),  dgamma = sum over rows of dy h,  dbeta = sum of dy
//
// A row is read once: LANES lanes have it in registers, eight neighbours at a time, so the variance is that of the distances from the
// mean and not a difference of two large sums.  The mean is a sum's first, which is off by the roundings of a sum as large as the values, and the mean of the
// distances from it: a row of one value has that mean exactly, and distances and a variance of 0 (see `centred`).  The next row's loads are on their way while a row is summed.  Memory bounds both passes: 16,384 rows of 4,096 in bf16
// forward 58 us, 4.6 TB/s (a large copy has 5.2); backward 393,216 rows of 160 85 us, 4.5 TB/s, of which 5 join the chunks' sums, and the vector ALU
// is busy for about half of it.
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
constexpr int norm_threads(int lanes) { return lanes <= 256 ? 256 : lanes; }
constexpr int norm_teams(int lanes) { return norm_threads(lanes) / lanes; }
// The same for the backward pass with its sums: the fewer workgroups, the fewer sums to join.  us with 512 threads and 256: 32,768 rows of 1,024 51 and 55,
// 8,192 of 4,096 56 and 60, 393,216 of 160 86 and 87; but 786,432 of 36 55 and 51.
constexpr int norm_grad_threads(int lanes, int eights) { return eights == 1 ? 256 : 512; }
constexpr int norm_grad_teams(int lanes, int eights) { return norm_grad_threads(lanes, eights) / lanes; }
// Sums of a workgroup's features that meet in LDS: those of each wave, or of each team of several waves.
constexpr int norm_grad_shares(int lanes, int eights) { return lanes <= 64 ? norm_grad_threads(lanes, eights) / 64 : norm_grad_teams(lanes, eights); }

// Sums over a row's lanes, the same in all of them, of a workgroup with one row.
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float (*meet)[16], int turn) {
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) meet[turn][threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) s += meet[turn][w];
    return s;
}

// The weights of a group's features in LDS, for registers are what decides how many rows are on their way: first halves of all eights, then second
// halves, so that neighbouring lanes read neighbouring 16 bytes, then the rest.
struct Weights {
    float* at;
    int eights;

    static __host__ __device__ constexpr size_t values(int features) { return (size_t)features / 8 * 8 + 8; }
    // Where feature f stands.
    static __device__ __forceinline__ int place(int f, int eights) {
        const int c = f >> 3;
        return c == eights ? f : 4 * (f & 4 ? eights + c : c) + (f & 3);
    }
    __device__ __forceinline__ void fill(float* lds, const float* from, int features, float none) {
        at = lds;
        eights = features >> 3;
        for (int c = threadIdx.x; c < eights; c += blockDim.x) {
            Eight<Fp32> w;
            if (from) w.load8(from + 8 * c);
            const uint32_t bits = as_bits(none);
            if (!from) w.words[0] = w.words[1] = u32x4{bits, bits, bits, bits};
            *reinterpret_cast<u32x4*>(at + 4 * c) = w.words[0];
            *reinterpret_cast<u32x4*>(at + 4 * (eights + c)) = w.words[1];
        }
        const int f = 8 * eights + threadIdx.x;
        if (f < features) at[f] = from ? from[f] : none;
    }
    // Of eight c (WIDE 8), or of feature c behind the last (WIDE 1).
    template <int WIDE>
    __device__ __forceinline__ Eight<Fp32> get(int c) const {
        Eight<Fp32> w;
        if constexpr (WIDE == 8) {
            w.words[0] = *reinterpret_cast<const u32x4*>(at + 4 * c);
            w.words[1] = *reinterpret_cast<const u32x4*>(at + 4 * (eights + c));
        } else {
            w.one(at[8 * eights + c]);
        }
        return w;
    }
};

// Mean and variance of a row over several waves by those of each wave's part: sums q of squares about a part's own mean m, of n values,
// make one of sum (q + n (m - mean)^2).
template <int TEAMS, int WAVES>
struct Parts {
    float size[WAVES], inverse[WAVES];
    float mean[2][TEAMS][WAVES], squares[2][TEAMS][WAVES];
};

// The mean of n values and the sum of their squares about it, from a first mean, the sum `rest` of the distances from it and the sum of those' squares: the
// mean is off by rest / n, which adds rest^2 / n to the squares.  Where that is not a small part of them (rows whose values are nearly one
// value, far from 0), what would be left of the squares is their rounding: they are summed again, by again(mean), which every lane of the wave calls.
template <class F>
__device__ __forceinline__ void centred(float& mean, float& squares, float rest, float inverse, F&& again) {
    const float off = rest * inverse;
    const bool anew = !(64.0f * off * rest < squares);      // (also where squares about the first mean are infinite)
    mean += off;
    squares -= rest * off;
    if (__any(anew)) {
        const float s = again(mean);
        squares = anew ? s : squares;       // a row's result does not hang on those beside it
    }
}

template <class X, class Y, int LANES, int N>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_kernel(Norm a) {
    constexpr int kTeams = norm_teams(LANES), kWaves = LANES <= 64 ? 1 : LANES / 64;
    using R = Row<X, LANES, N>;
    __shared__ Parts<kTeams, kWaves> parts;
    extern __shared__ __align__(16) float norm_weights[];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES, wave = lane >> 6, n = (int)(ch.hi - ch.lo), features = a.features;
    R x, next;
    x.load(a.x, (size_t)(ch.lo + team) * a.ldx, lane, Extent(features, team < n));
    Weights gamma, beta;
    gamma.fill(norm_weights, a.gamma ? a.gamma + (size_t)ch.group * features : nullptr, features, 1.0f);
    beta.fill(norm_weights + Weights::values(features), a.beta ? a.beta + (size_t)ch.group * features : nullptr, features, 0.0f);
    if (kWaves > 1 && (int)threadIdx.x < kWaves) {
        int size = threadIdx.x == 0 ? features & 7 : 0;
        for (int i = 0; i < N; ++i) {
            const int left = (features >> 3) - (64 * (int)threadIdx.x + LANES * i);
            size += 8 * (left < 0 ? 0 : left > 64 ? 64 : left);
        }
        parts.size[threadIdx.x] = (float)size;
        parts.inverse[threadIdx.x] = size ? 1.0f / (float)size : 0.0f;
    }
    __syncthreads();
    const float own = kWaves > 1 ? parts.inverse[wave] : a.inverse;
    auto step = [&](R& x, R& next, int r0, int turn) {
        const Extent w(features, r0 + team < n);
        next.load(a.x, (size_t)(ch.lo + r0 + kTeams + team) * a.ldx, lane, Extent(features, r0 + kTeams + team < n));
        constexpr int kGroup = LANES < 64 ? LANES : 64;
        float sum = 0.0f, rest = 0.0f, squares = 0.0f;
        R::each(lane, w, [&](auto wide, auto i) {
#pragma unroll
            for (int e = 0; e < wide; ++e) sum += x.at(i).get(e);
        });
        float mean = lanes_sum<kGroup>(sum) * own;         // of the wave's part
        R::each(lane, w, [&](auto wide, auto i) {
#pragma unroll
            for (int e = 0; e < wide; ++e) {
                const float d = x.at(i).get(e) - mean;
                rest += d;
                squares = __builtin_fmaf(d, d, squares);
            }
        });
        squares = lanes_sum<kGroup>(squares);
        centred(mean, squares, lanes_sum<kGroup>(rest), own, [&](float mean) {
            float s = 0.0f;
            R::each(lane, w, [&](auto wide, auto i) {
#pragma unroll
                for (int e = 0; e < wide; ++e) {
                    const float d = x.at(i).get(e) - mean;
                    s = __builtin_fmaf(d, d, s);
                }
            });
            return lanes_sum<kGroup>(s);
        });
        if constexpr (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) {
                parts.mean[turn][team][wave] = mean;
                parts.squares[turn][team][wave] = squares;
            }
            __syncthreads();
            // the mean by the parts' distances from the first one's: of equal ones it is that one
            const float first = parts.mean[turn][team][0];
            rest = squares = 0.0f;
#pragma unroll
            for (int k = 1; k < kWaves; ++k) rest = __builtin_fmaf(parts.size[k], parts.mean[turn][team][k] - first, rest);
            mean = __builtin_fmaf(rest, a.inverse, first);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float d = parts.mean[turn][team][k] - mean;
                squares += __builtin_fmaf(parts.size[k] * d, d, parts.squares[turn][team][k]);
            }
        }
        const float scale = __builtin_amdgcn_rsqf(squares * a.inverse + a.eps);     // the hardware's: within a step of fp32
        x.forget();
        const size_t row = (size_t)(ch.lo + r0 + team);
        if (a.stats && lane == 0 && r0 + team < n) {
            a.stats[2 * row] = mean;
            a.stats[2 * row + 1] = scale;
        }
        Row<Y, LANES, N> y;
        R::each(lane, w, [&](auto wide, auto i) {
            const int c = i < N ? lane + LANES * i : lane;
            const Eight<Fp32> g = gamma.get<wide>(c), b = beta.get<wide>(c);
            float v[8] = {};
#pragma unroll
            for (int e = 0; e < wide; ++e) v[e] = __builtin_fmaf(g.get(e), (x.at(i).get(e) - mean) * scale, b.get(e));
            y.at(i).set(v);
            y.store(i, a.y, row * a.ldy, lane, w);
        });
    };
    for (int r0 = 0; r0 < n; r0 += 2 * kTeams) {
        step(x, next, r0, 0);
        if (r0 + kTeams >= n) break;
        step(next, x, r0 + kTeams, 1);
    }
}

// The whole backward pass, every row read once: a lane has its features' sums in registers to the end of the chunk.
template <class X, class Y, int LANES, int N>
__global__ __launch_bounds__(norm_grad_threads(LANES, N)) void layer_norm_grad_kernel(Norm a) {
    constexpr int kTeams = norm_grad_teams(LANES, N), kWaves = LANES <= 64 ? 1 : LANES / 64;
    // 512 threads have 256 registers each at most: four eights a lane of fp32, with the sums, leave no room for the next row
    constexpr bool kAhead = LANES < 512 || N < 4 || !kIs32<Y>;
    using R = Row<X, LANES, N>;
    __shared__ float meet[2][kTeams][2][kWaves];
    extern __shared__ __align__(16) float norm_weights[];
    const Chunk ch = norm_chunk(a, blockIdx.x, a.dgamma != nullptr);
    if (ch.group < 0 || (a.dgamma && ch.count > 1 && ch.shared >= a.shared_max)) return;    // (the second only with offsets that fall)
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES, wave = lane >> 6, n = (int)(ch.hi - ch.lo), features = a.features;
    struct Held {
        R x;
        Row<Y, LANES, N> dy;
        float mean, scale;
    } held, then;
    auto load = [&](Held& h, int r) {
        const Extent w(features, r < n);
        const size_t row = (size_t)(ch.lo + r);
        h.x.load(a.x, row * a.ldx, lane, w);
        h.dy.load(a.dy, row * a.lddy, lane, w);
        h.mean = h.scale = 0.0f;
        if (r < n) {
            h.mean = a.stats[2 * row];
            h.scale = a.stats[2 * row + 1];
        }
    };
    load(held, team);
    Weights gamma;
    gamma.fill(norm_weights, a.gamma ? a.gamma + (size_t)ch.group * features : nullptr, features, 1.0f);
    __syncthreads();
    Sums<LANES, N> dg, db;
    dg.clear();
    db.clear();
    auto step = [&](Held& h, Held& next, int r0, int turn) {
        const Extent w(features, r0 + team < n);
        if (kAhead) load(next, r0 + kTeams + team);
        const float mean = h.mean, scale = h.scale;
        float s1 = 0.0f, s2 = 0.0f;
        R::each(lane, w, [&](auto wide, auto i) {
            const Eight<Fp32> g = gamma.get<wide>(i < N ? lane + LANES * i : lane);
#pragma unroll
            for (int e = 0; e < wide; ++e) {
                const float d = h.dy.at(i).get(e), x = (h.x.at(i).get(e) - mean) * scale, u = d * g.get(e);
                s1 += u;
                s2 = __builtin_fmaf(u, x, s2);
                dg.at(i)[e] = __builtin_fmaf(d, x, dg.at(i)[e]);
                db.at(i)[e] += d;
            }
        });
        s1 = lanes_sum<(LANES < 64 ? LANES : 64)>(s1);
        s2 = lanes_sum<(LANES < 64 ? LANES : 64)>(s2);
        if constexpr (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) {
                meet[turn][team][0][wave] = s1;
                meet[turn][team][1][wave] = s2;
            }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                s1 += meet[turn][team][0][k];
                s2 += meet[turn][team][1][k];
            }
        }
        h.x.forget();
        h.dy.forget();
        if (a.y) {
            // in the formula's order: with scale taken into the means, its square would leave fp32's range long before dx does (scale is up to 2^63)
            const float m1 = -(s1 * a.inverse), m2 = -(s2 * a.inverse);
            R dx;
            R::each(lane, w, [&](auto wide, auto i) {
                const Eight<Fp32> g = gamma.get<wide>(i < N ? lane + LANES * i : lane);
                float v[8] = {};
#pragma unroll
                for (int e = 0; e < wide; ++e) v[e] = scale * __builtin_fmaf((h.x.at(i).get(e) - mean) * scale, m2, __builtin_fmaf(h.dy.at(i).get(e), g.get(e), m1));
                dx.at(i).set(v);
                dx.store(i, a.y, (size_t)(ch.lo + r0 + team) * a.ldy, lane, w);
            });
        }
        if (!kAhead) load(next, r0 + kTeams + team);
    };
    for (int r0 = 0; r0 < n; r0 += 2 * kTeams) {
        step(held, kAhead ? then : held, r0, 0);
        if (r0 + kTeams >= n) break;
        step(kAhead ? then : held, held, r0 + kTeams, 1);
    }
    if (!a.dgamma) return;
    float* to = ch.count == 1 ? a.dgamma + (size_t)ch.group * features : a.partial + (size_t)ch.shared * 2 * features;
    float* to_beta = ch.count == 1 ? a.dbeta + (size_t)ch.group * features : to + features;
    const Extent all(features, true);
    if constexpr (LANES > 64 && kTeams == 1) {
        R::each(lane, all, [&](auto, auto i) {
            Row<Fp32, LANES, N> out;
            out.at(i).set(dg.at(i));
            out.store(i, to, 0, lane, all);
            out.at(i).set(db.at(i));
            out.store(i, to_beta, 0, lane, all);
        });
    } else {
        // the rows of a wave by exchanges, then those of the waves or teams, kShares of them, through LDS (where the weights were)
        constexpr int kShares = norm_grad_shares(LANES, N);
        const int share = LANES <= 64 ? threadIdx.x >> 6 : team;
        if constexpr (LANES < 64) {
            dg.sum_groups();
            db.sum_groups();
        }
        __syncthreads();
        const int pitch = (int)Weights::values(features);
        if (LANES >= 64 || (int)(threadIdx.x & 63) < LANES)
            R::each(lane, all, [&](auto wide, auto i) {
                float* at = norm_weights + 2 * share * pitch;
                const float (&g)[8] = dg.at(i), (&b)[8] = db.at(i);
                if constexpr (wide == 8) {
                    const int c = lane + LANES * i;
                    *reinterpret_cast<f32x4*>(at + 4 * c) = f32x4{g[0], g[1], g[2], g[3]};
                    *reinterpret_cast<f32x4*>(at + 4 * (all.eights + c)) = f32x4{g[4], g[5], g[6], g[7]};
                    *reinterpret_cast<f32x4*>(at + pitch + 4 * c) = f32x4{b[0], b[1], b[2], b[3]};
                    *reinterpret_cast<f32x4*>(at + pitch + 4 * (all.eights + c)) = f32x4{b[4], b[5], b[6], b[7]};
                } else {
                    at[8 * all.eights + lane] = g[0];
                    at[pitch + 8 * all.eights + lane] = b[0];
                }
            });
        __syncthreads();
        for (int f = threadIdx.x; f < features; f += norm_grad_threads(LANES, N)) {
            const int at = Weights::place(f, all.eights);
            float g = 0.0f, b = 0.0f;
#pragma unroll
            for (int k = 0; k < kShares; ++k) {
                g += norm_weights[2 * k * pitch + at];
                b += norm_weights[2 * k * pitch + pitch + at];
            }
            to[f] = g;
            to_beta[f] = b;
        }
    }
}

// Rows that do not fit the registers of a workgroup (more than 16,391 features) are read again for each sum, from L2 or behind it: 1024 threads a row.  2,048 rows of
// 30,000 in bf16: 87 us forward, 2.8 TB/s; 1,024 of them backward 106 us with the sums, which read them once more.
constexpr int kLongThreads = 1024;

template <class X, class Y>
__global__ __launch_bounds__(kLongThreads) void layer_norm_long_kernel(Norm a) {
    __shared__ float meet[4][16];
    const Chunk ch = norm_chunk(a, blockIdx.x, false);
    if (ch.group < 0) return;
    const float* gamma = a.gamma ? a.gamma + (size_t)ch.group * a.features : nullptr;
    const float* beta = a.beta ? a.beta + (size_t)ch.group * a.features : nullptr;
    for (int64_t row = ch.lo; row < ch.hi; ++row) {
        const size_t at = (size_t)row * a.ldx;
        float sum = 0.0f, rest = 0.0f, squares = 0.0f;
        auto each = [&](auto f) {
            for (int c = 8 * threadIdx.x; c < a.features; c += 8 * kLongThreads) {
                Eight<X> x;
                x.load(a.x, at + c, a.features - c);
#pragma unroll
                for (int e = 0; e < 8; ++e) f(x.get(e), c + e < a.features);
            }
        };
        each([&](float v, bool) { sum += v; });     // zeros behind the last
        float mean = row_sum<kLongThreads>(sum, meet, 0) * a.inverse;
        each([&](float v, bool there) {
            const float d = there ? v - mean : 0.0f;
            rest += d;
            squares = __builtin_fmaf(d, d, squares);
        });
        rest = row_sum<kLongThreads>(rest, meet, 1);
        squares = row_sum<kLongThreads>(squares, meet, 2);
        centred(mean, squares, rest, a.inverse, [&](float mean) {       // the same sums in all waves
            float s = 0.0f;
            each([&](float v, bool there) {
                const float d = there ? v - mean : 0.0f;
                s = __builtin_fmaf(d, d, s);
            });
            return row_sum<kLongThreads>(s, meet, 3);
        });
        const float scale = 1.0f / sqrtf(squares * a.inverse + a.eps);
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
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(gamma ? w.get(e) : 1.0f, (x.get(e) - mean) * scale, beta ? b.get(e) : 0.0f);
            y.set(v);
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
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float u = dy.get(e) * (gamma ? w.get(e) : 1.0f), h = (x.get(e) - mean) * scale;
                    if (pass == 0) {
                        s1 += f + e < a.features ? u : 0.0f;
                        s2 += f + e < a.features ? u * h : 0.0f;
                    }
                    v[e] = scale * (u - s1 - h * s2);
                }
                dx.set(v);
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
constexpr int kJoinThreads = 1024, kJoinSlices = kJoinThreads / 16;

__global__ __launch_bounds__(kJoinThreads) void layer_norm_join_kernel(Norm a) {
    __shared__ __align__(16) f32x4 slices[kJoinSlices][16];
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
    // 64 values a workgroup, four a thread; 64 slices of it have every 64th chunk
    const int all = 2 * a.features, slice = threadIdx.x >> 4, e0 = 4 * (threadIdx.x & 15);
    for (int b = 64 * blockIdx.x; b < all; b += 64 * gridDim.x) {
        const int e = b + e0, left = all - e;
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        const float* from = a.partial + (size_t)first * all + e;
        if (left >= 4) {
            typedef f32x4 at_four __attribute__((aligned(4)));
#pragma unroll 4
            for (uint32_t c = slice; c < count; c += kJoinSlices) s += *reinterpret_cast<const at_four*>(from + (size_t)c * all);
        } else if (left > 0) {
            for (uint32_t c = slice; c < count; c += kJoinSlices) {
                s[0] += from[(size_t)c * all];
                if (left > 1) s[1] += from[(size_t)c * all + 1];
                if (left > 2) s[2] += from[(size_t)c * all + 2];
            }
        }
        slices[slice][threadIdx.x & 15] = s;
        __syncthreads();
        if (threadIdx.x < 64) {
            float sum = 0.0f;
            for (int k = 0; k < kJoinSlices; ++k) sum += slices[k][threadIdx.x >> 2][threadIdx.x & 3];
            const int f = b + threadIdx.x;
            if (f < a.features) a.dgamma[(size_t)g * a.features + f] = sum;
            else if (f < all) a.dbeta[(size_t)g * a.features + (f - a.features)] = sum;
        }
        __syncthreads();
    }
}

}  // namespace pcc_train
