// The activations of the head's products and their slopes.
#pragma once

#include "rows.cuh"

namespace eprow {

// The upper tail of the normal distribution at |z|, over exp(-z^2 / 2): a polynomial in t = 1 / (1 + 0.35 |z|), fitted
// (weighted least squares, reweighted towards the largest error) to 1.1e-7 (1 + z^2) of the tail itself up to |z| = 14,
// where fp32 loses as much by rounding the exponential's argument.  The gradient needs the same exponential, and where the
// slope of z Phi(z) crosses zero the exponential is a common factor of the terms that cancel.
// For z = (z0, z1): the bell exp(-z^2 / 2), |z| and that tail.
__device__ __forceinline__ void normal_parts(float z0, float z1, Pair &bell, Pair &size, Pair &tail) {
    const Pair z(z0, z1);
    size = Pair(fabsf(z0), fabsf(z1));
    float a, b;
    fma2(size, Pair(0.35f), Pair(1.f)).get(a, b);
    const Pair t(reciprocal_fast(a), reciprocal_fast(b));
    Pair q = fma2(t, Pair(0.0452263094f), Pair(-0.186698169f));
    q = fma2(q, t, Pair(0.214374468f));
    q = fma2(q, t, Pair(0.00660444144f));
    q = fma2(q, t, Pair(0.143951952f));
    q = fma2(q, t, Pair(0.136762664f));
    q = fma2(q, t, Pair(0.139778391f));
    tail = mul2(q, t);
    mul2(mul2(z, z), Pair(-0.5f * 1.44269504f)).get(a, b);
    bell = Pair(exp2_fast(a), exp2_fast(b));
}
// q bell below zero, 1 - q bell above: Phi(z) and the slope of z Phi(z) from what they are at -|z|.  Chosen, not computed
// from one another: 1 - (1 - m) would leave nothing of a small m.
__device__ __forceinline__ Pair either_side(float z0, float z1, Pair q, Pair bell) {
    float low0, low1, high0, high1;
    const Pair m = mul2(q, bell);
    m.get(low0, low1);
    fma2(m, Pair(-1.f), Pair(1.f)).get(high0, high1);
    return Pair(z0 >= 0.f ? high0 : low0, z1 >= 0.f ? high1 : low1);
}
__device__ __forceinline__ void gelu2(float &v0, float &v1) {
    Pair bell, size, tail;
    normal_parts(v0, v1, bell, size, tail);
    mul2(Pair(v0, v1), either_side(v0, v1, tail, bell)).get(v0, v1);
}
// v *= slope of GELU at z
__device__ __forceinline__ void times_gelu_slope2(float &v0, float &v1, float z0, float z1) {
    Pair bell, size, tail;
    normal_parts(z0, z1, bell, size, tail);
    const Pair q = fma2(size, Pair(-0.39894228f), tail);
    mul2(Pair(v0, v1), either_side(z0, z1, q, bell)).get(v0, v1);
}

// act(z) of n values; the switch is outside the loops, and taken by all threads alike.
template <int n>
__device__ __forceinline__ void activate(float (&v)[n], int act) {
    if (act == EP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v[i]));   // (a NaN stays one)
    } else if (act == EP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i + 1 < n; i += 2) gelu2(v[i], v[i + 1]);
        if constexpr (n % 2 == 1) {
            float none = 0.f;
            gelu2(v[n - 1], none);
        }
    } else if (act == EP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] *= reciprocal_fast(1.f + exp_fast(-v[i]));   // (1 / infinity: far below zero the sigmoid is 0)
    }
}
// v *= act'(z)
template <int n>
__device__ __forceinline__ void times_slope(float (&v)[n], const float (&z)[n], int act) {
    if (act == EP_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = z[i] > 0.f ? v[i] : 0.f;
    } else if (act == EP_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < n; i += 2) times_gelu_slope2(v[i], v[i + 1], z[i], z[i + 1]);
    } else if (act == EP_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float s = reciprocal_fast(1.f + exp_fast(-z[i]));
            v[i] *= s * fmaf(z[i], 1.f - s, 1.f);
        }
    }
}

}  // namespace eprow
