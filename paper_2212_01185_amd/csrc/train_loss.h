// Code length of a pixel under the mixture its head outputs describe, and its gradient.
//
// For a component with a = (x - 1/2)/256 and b = (x + 1/2)/256 in units of its width, q = F(b) - F(a) is its probability of
// level x, and with the density f:  dq/dmu = (f(a) - f(b)) / sigma,  dq/dlog sigma = a f(a) - b f(b).
// A difference of two values of F next to each other loses what a code length needs (the coder's rule adds one count of
// 65,536, so q matters down to 1e-5 and below), so nothing here subtracts two such values:
//   - the component is mirrored so that its middle m is right of the mean, and upper tails are used: near = m - h,
//     far = m + h, half a level is h = 1 / (512 sigma)
//   - logistic: S(z) = 1 / (1 + e^z);  S(near) - S(far) = S(near) (1 - S(far)) (1 - e^-2h),
//     f(near) - f(far) = q (1 - S(near) - S(far))
//   - Gaussian, levels narrow against the curvature (2h (m + 1) < 1/2): the derivatives of the density are Hermite
//     polynomials, q = 2h f(m) (1 + He2 D2/24 + He4 D4/1920), f(near) - f(far) = 2h f(m) (He1 + He3 D2/24 + He5 D4/1920) with
//     D = 2h; what is left out is below D^6 (m + 1)^6 / 322,560 < 5e-8
//   - Gaussian, else: tails as f(z) R(z), Mills' ratio R a polynomial in 1 / (1 + z/4) (fitted: 4e-8 apart, 4e-7 in fp32);
//     the two differ by a factor of e^(1/2) at least, or lie near the mean
//   - near f(near) - far f(far) = m (f(near) - f(far)) - h (f(near) + f(far))
#pragma once

#include <type_traits>

#include "train_device.h"

namespace pcc_train {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }
// The same for |v| <= 8, with what the rounding of v log2(e) and of the constant left out: without it e^-8 is 3e-7 off, and a
// distance in widths of that component with it.
__device__ __forceinline__ float exp_exact(float v) {
    const float t = v * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, __builtin_fmaf(v, 1.925962989e-8f, __builtin_fmaf(v, kLog2e, -t)) * kLn2, e);
}
// f(z) of the standard normal distribution.
__device__ __forceinline__ float normal_density(float z) { return 0.39894228040143268f * __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e)); }

// Q(z) / f(z) of the standard normal distribution, z >= 0.
__device__ __forceinline__ float mills(float z) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.25f, z, 1.0f));
    float p = 4.959281161e-02f;
    p = __builtin_fmaf(p, t, -2.027588040e-01f);
    p = __builtin_fmaf(p, t, 2.396807224e-01f);
    p = __builtin_fmaf(p, t, -7.955849171e-02f);
    p = __builtin_fmaf(p, t, 1.597021073e-01f);
    p = __builtin_fmaf(p, t, 1.478174478e-01f);
    p = __builtin_fmaf(p, t, 2.045509815e-01f);
    p = __builtin_fmaf(p, t, 2.342851609e-01f);
    p = __builtin_fmaf(p, t, 2.500021756e-01f);
    p = __builtin_fmaf(p, t, 2.499999851e-01f);
    return p * t;
}

constexpr float kFar = 0x1p40f;

struct Bin {
    float q;        // probability of the level
    float d_mu;     // f(a) - f(b)
    float d_ls;     // a f(a) - b f(b)
};

// v, or -v where `sign` is negative.
__device__ __forceinline__ float with_sign(float v, float sign) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, v) ^ (__builtin_bit_cast(uint32_t, sign) & 0x80000000u));
}

// mid: the level's middle, h: half a level, both in widths of the component; first, last: the level is 0, 255 (open ends).
template <int DIST>
__device__ __forceinline__ Bin bin_of(float mid, float h, bool first, bool last) {
    const bool mirrored = __builtin_signbit(mid);
    // further than kFar nothing is left of the component; an infinite distance would make m (f(near) - f(far)) inf * 0 (a NaN stays one)
    const float m = fabsf(mid) > kFar ? kFar : fabsf(mid), near = m - h, far = m + h;
    const bool open_near = mirrored ? last : first, open_far = mirrored ? first : last;
    float q, diff, sum;     // diff, sum: f(near) -+ f(far)
    if (DIST == 1) {
        const float en = exp_of(near), ef = exp_of(-far);
        const float sn = open_near ? 1.0f : __builtin_amdgcn_rcpf(1.0f + en);
        const float sf = open_far ? 0.0f : ef * __builtin_amdgcn_rcpf(1.0f + ef);
        const float d = 2.0f * h;
        const float gap = d < 0.1f ? d * __builtin_fmaf(d, __builtin_fmaf(d, __builtin_fmaf(d, -1.0f / 24.0f, 1.0f / 6.0f), -0.5f), 1.0f)
                                   : 1.0f - exp_of(-d);
        const float both = 1.0f - sn - sf;
        if (open_near || open_far) {
            q = open_near ? __builtin_amdgcn_rcpf(1.0f + ef) : sn;
            const float fn = open_near ? 0.0f : sn * (1.0f - sn), ff = sf * (1.0f - sf);
            diff = fn - ff;
            sum = fn + ff;
        } else {
            q = sn * (1.0f - sf) * gap;
            diff = q * both;
            sum = __builtin_fmaf(sn, 1.0f - sn, sf * (1.0f - sf));
        }
    } else {
        const float d = 2.0f * h;
        if (d * (m + 1.0f) < 0.5f && !open_near && !open_far) {
            const float f = normal_density(m), z2 = m * m, d2 = d * d * (1.0f / 24.0f), d4 = d * d * d * d * (1.0f / 1920.0f);
            const float he2 = z2 - 1.0f, he4 = __builtin_fmaf(z2, z2 - 6.0f, 3.0f), he6 = __builtin_fmaf(z2, __builtin_fmaf(z2, z2 - 15.0f, 45.0f), -15.0f);
            const float he3 = m * (z2 - 3.0f), he5 = m * __builtin_fmaf(z2, z2 - 10.0f, 15.0f);
            const float df = d * f;
            Bin b;
            b.q = df * __builtin_fmaf(he4, d4, __builtin_fmaf(he2, d2, 1.0f));
            const float dm = df * __builtin_fmaf(he5, d4, __builtin_fmaf(he3, d2, m));
            b.d_mu = with_sign(dm, mid);
            b.d_ls = df * __builtin_fmaf(he6, d4, __builtin_fmaf(he4, d2, he2));
            return b;
        }
        const float fn = open_near ? 0.0f : normal_density(near), ff = open_far ? 0.0f : normal_density(far);
        const float tn = fn * mills(fabsf(near)), tail_near = open_near ? 1.0f : near < 0.0f ? 1.0f - tn : tn;
        const float tail_far = open_far ? 0.0f : ff * mills(far);
        q = tail_near - tail_far;
        diff = fn - ff;
        sum = fn + ff;
    }
    return {q, with_sign(diff, mid), __builtin_fmaf(m, diff, -(h * sum))};
}

// One channel: returns its bits and puts the gradient in place of the channel's 3 K outputs (logits, means, log-sigmas).  shift: what
// the coupling adds to the means.  A level's distance from a mean is taken in 64 bits: in 32 the sum of mean and coupling is rounded
// by 3e-8, a ten-thousandth of the narrowest component's width.
template <int K, int DIST>
__device__ __forceinline__ float channel_loss(float (&o)[3 * K], const double (&shift)[K], int level, float factor) {
    float top = o[0];
#pragma unroll
    for (int k = 1; k < K; ++k) top = fmaxf(top, o[k]);
    float pi[K], total = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) { pi[k] = exp_of(o[k] - top); total += pi[k]; }
    const float inverse = __builtin_amdgcn_rcpf(total);
    const double x = (double)level * (1.0 / 256.0);
    float p = 0.0f, q[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        pi[k] *= inverse;
        const float raw = o[2 * K + k];
        const bool inside = raw >= -8.0f && raw <= 4.0f;
        const float ls = raw > 4.0f ? 4.0f : raw >= -8.0f ? raw : -8.0f;
        const float width = exp_exact(-ls);
        const Bin b = bin_of<DIST>((float)(x - (double)o[K + k] - shift[k]) * width, width * (1.0f / 512.0f), level == 0, level == 255);
        q[k] = b.q;
        p = __builtin_fmaf(pi[k], b.q, p);
        o[K + k] = pi[k] * b.d_mu * width;
        o[2 * K + k] = inside ? pi[k] * b.d_ls : 0.0f;
    }
    const float counts = __builtin_fmaf(65280.0f, p, 1.0f);
    const float outer = factor * (-65280.0f / kLn2) * __builtin_amdgcn_rcpf(counts);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        o[k] = outer * pi[k] * (q[k] - p);
        o[K + k] *= outer;
        o[2 * K + k] *= outer;
    }
    return 16.0f - __builtin_amdgcn_logf(counts);
}

// A lane has a pixel.  A pixel's 12 K outputs are neighbours in memory, so a wave brings its 64 pixels' to LDS 16 bytes a lane, each lane
// takes its own from there (rows of 12 K values: the 16 lanes that are served together read different banks), and the
// gradients go the same way back.  Nothing is shared between waves.  2048x1365 pixels, K = 5, gradients in bf16: 202 us, 5.1 TB/s, what a large copy
// has (each lane reading its own row from memory: 821; with a division for each piece, and both 16-bit types in one kernel: 386).
// One wave is a workgroup (2048x1365 pixels, K = 5: 202 us; four are 208).  The vector ALU is busy for 90 % of that time.  K = 3 takes 112 us, K = 7 287
// (4.98 TB/s) and with fp32 gradients 429 (4.4: 21.5 KB of LDS for a wave leave seven of them on a compute unit); logistic 113, 190, 253 and 360; bits
// alone 92, 170 and 369 us (their floors are 82, 134 and 186: the gradients are computed all the same).
constexpr int kLossWaves = 1;

// GRAD: the gradients' type.
template <int K, int DIST, int GRAD>
__global__ __launch_bounds__(64 * kLossWaves) void mixture_loss_kernel(const float* params, size_t ldp, const uint8_t* __restrict__ rgb,
                                                                       const float* __restrict__ weight, size_t count, float scale,
                                                                       float* __restrict__ bits, void* grad, size_t ldg) {
    constexpr int N = 12 * K, kPieces = 3 * K;       // 16-byte pieces of a row
    typedef f32x4 at_four __attribute__((aligned(4)));
    typedef u16x4 at_four_16 __attribute__((aligned(4)));
    extern __shared__ __align__(16) float loss_shared[];
    const int lane = threadIdx.x & 63;
    float* lds = loss_shared + (threadIdx.x >> 6) * 64 * N;
    const size_t i0 = (size_t)blockIdx.x * (64 * kLossWaves) + uniform(threadIdx.x & ~63u), i = i0 + lane;
    if (i0 >= count) return;
    const int pixels = count - i0 < 64 ? (int)(count - i0) : 64;
    const float* from = params + i0 * ldp;
    // 64 whole rows one behind the other are one piece of memory; else every piece has its row looked up
    const bool in_line = pixels == 64 && ldp == (size_t)N, out_line = pixels == 64 && ldg == (size_t)N;
    if (in_line) {
#pragma unroll
        for (int s = 0; s < kPieces; ++s) *reinterpret_cast<f32x4*>(lds + 4 * (lane + 64 * s)) = *reinterpret_cast<const at_four*>(from + 4 * (lane + 64 * s));
    } else {
        for (int s = 0; s < kPieces; ++s) {
            const int id = lane + 64 * s, r = id / kPieces, c = id % kPieces;
            if (r < pixels) *reinterpret_cast<f32x4*>(lds + 4 * id) = *reinterpret_cast<const at_four*>(from + (size_t)r * ldp + 4 * c);
        }
    }
    const bool mine = lane < pixels;
    const float wt = !mine ? 0.0f : weight ? weight[i] : 1.0f;
    const int rgb3[3] = {mine ? rgb[3 * i] : 0, mine ? rgb[3 * i + 1] : 0, mine ? rgb[3 * i + 2] : 0};
    const float rh = (float)rgb3[0] * (1.0f / 256.0f), gh = (float)rgb3[1] * (1.0f / 256.0f);
    __builtin_amdgcn_wave_barrier();

    float o[N], sum = 0.0f;
    const f32x4* row = reinterpret_cast<const f32x4*>(lds + lane * N);
#pragma unroll
    for (int s = 0; s < kPieces; ++s) {
        const f32x4 v = row[s];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[4 * s + e] = v[e];
    }
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        float ch[3 * K];
        double shift[K];
#pragma unroll
        for (int j = 0; j < 3 * K; ++j) ch[j] = o[3 * K * c + j];
#pragma unroll
        for (int k = 0; k < K; ++k)
            shift[k] = c == 0 ? 0.0 : c == 1 ? (double)o[9 * K + k] * rh : __builtin_fma((double)o[11 * K + k], (double)gh, (double)o[10 * K + k] * rh);
        sum += channel_loss<K, DIST>(ch, shift, rgb3[c], wt * scale);
#pragma unroll
        for (int j = 0; j < 3 * K; ++j) o[3 * K * c + j] = ch[j];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float d = ch[K + k];
            if (c == 1) o[9 * K + k] = d * rh;
            if (c == 2) { o[10 * K + k] = d * rh; o[11 * K + k] = d * gh; }
        }
    }
    if (__ballot(wt == 0.0f)) {             // pixels that do not count, whatever their outputs were
        if (wt == 0.0f) sum = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] = wt == 0.0f ? 0.0f : o[j];
    }
    if (bits && mine) bits[i] = sum;
    if (!grad) return;
    __builtin_amdgcn_wave_barrier();        // every lane has its outputs: LDS is free for the gradients
    if constexpr (GRAD == PCC_FP32) {
        f32x4* to = reinterpret_cast<f32x4*>(lds + lane * N);
#pragma unroll
        for (int s = 0; s < kPieces; ++s) to[s] = f32x4{o[4 * s], o[4 * s + 1], o[4 * s + 2], o[4 * s + 3]};
        __builtin_amdgcn_wave_barrier();
        float* out = static_cast<float*>(grad) + i0 * ldg;
        if (out_line) {
#pragma unroll
            for (int s = 0; s < kPieces; ++s) *reinterpret_cast<at_four*>(out + 4 * (lane + 64 * s)) = *reinterpret_cast<const f32x4*>(lds + 4 * (lane + 64 * s));
        } else {
            for (int s = 0; s < kPieces; ++s) {
                const int id = lane + 64 * s, r = id / kPieces, c = id % kPieces;
                if (r < pixels) *reinterpret_cast<at_four*>(out + (size_t)r * ldg + 4 * c) = *reinterpret_cast<const f32x4*>(lds + 4 * id);
            }
        }
    } else {
        using T = std::conditional_t<GRAD == PCC_BF16, Bf16, Fp16>;
        u16x4* to = reinterpret_cast<u16x4*>(lds) + lane * kPieces;
#pragma unroll
        for (int s = 0; s < kPieces; ++s) to[s] = u16x4{to16<T>(o[4 * s]), to16<T>(o[4 * s + 1]), to16<T>(o[4 * s + 2]), to16<T>(o[4 * s + 3])};
        __builtin_amdgcn_wave_barrier();
        u16* out = static_cast<u16*>(grad) + i0 * ldg;
        const u16x4* held = reinterpret_cast<const u16x4*>(lds);
        const bool even = ldg % 2 == 0 && (reinterpret_cast<uintptr_t>(grad) & 3) == 0;
        if (out_line && even) {
#pragma unroll
            for (int s = 0; s < kPieces; ++s) *reinterpret_cast<at_four_16*>(out + 4 * (lane + 64 * s)) = held[lane + 64 * s];
        } else {
            for (int s = 0; s < kPieces; ++s) {
                const int id = lane + 64 * s, r = id / kPieces, c = id % kPieces;
                if (r >= pixels) continue;
                u16* at = out + (size_t)r * ldg + 4 * c;
                if (even) *reinterpret_cast<at_four_16*>(at) = held[id];
                else for (int e = 0; e < 4; ++e) at[e] = held[id][e];
            }
        }
    }
}

}  // namespace pcc_train
