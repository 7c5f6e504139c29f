// The activations of the dense product and their derivatives, of values in float.
#pragma once
#include "common.h"

namespace moe {

// Phi(z), and the root of exp(-z^2 / 2) on the way: erfc by the five-term rational approximation of Abramowitz & Stegun 7.1.26 (off by
// at most 1.5e-7), taken as it is on the negative side, where 1 - erf would lose what is left.  For results that are
// rounded to bfloat16.
__device__ __forceinline__ float normal_cdf_fast(float z, float* root) {
    const float x = fabsf(z) * 0.70710678118654752440f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
    *root = __builtin_amdgcn_exp2f(x * x * (-0.5f * 1.44269504088896340736f));
    float p = fmaf(t, 1.061405429f, -1.453152027f);
    p = fmaf(t, p, 1.421413741f);
    p = fmaf(t, p, -0.284496736f);
    p = fmaf(t, p, 0.254829592f);
    const float tail = 0.5f * p * t * *root * *root;
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(-0.70710678118654752440f * z); }

// z Phi(z) = max(z, 0) - |z| Phi(-|z|) in as few instructions as it takes: with 256 values to a lane they are a tenth of a GEMM's time over
// K = 2048.  Phi(-a) = exp(-a^2 / 2) Q(a), Q(a) = erfcx(a / sqrt 2) / 2 by six terms in t = 1 / (1 + 0.42 a), fitted on 0 <= a <= 14 by linear
// programming in 64 bits to the least e with an error of Q below e Q min(1 / Phi(-a), 1000): Phi(-a) is off by at most 8.8e-8 and by 8.8e-5 of
// itself, in float 9.7e-5, so that far on the negative side a result is within 0.03 of a half step of bfloat16 too.  (Five terms by the usual
// fit of the absolute error alone, one instruction less: 0.4 % of a result at -6, 2 % at -10.)
// (The maximum is a sum, which keeps a NaN; beyond 32 there is nothing to subtract, and an infinity stays one.)
__device__ __forceinline__ float gelu_tail_f(float z) {
    const float a = fminf(fabsf(z), 32.0f);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.42f, a, 1.0f));
    const float ex = __builtin_amdgcn_exp2f(a * (a * (-0.5f * 1.44269504088896340736f)));
    float p = fmaf(t, 0.05793207f, -0.23506184f);
    p = fmaf(t, p, 0.25901139f);
    p = fmaf(t, p, 0.07209909f);
    p = fmaf(t, p, 0.17923986f);
    p = fmaf(t, p, 0.16677961f);
    return fmaf(-a, p * (t * ex), fmaf(0.5f, fabsf(z), 0.5f * z));
}

// z sigmoid(z).  exp(-z) leaves the range of the reciprocal instruction at -87.3, and that of float soon after, where the result is 1e-36 still.
// bfloat16: such results are lost, and zero.  (The form that keeps them has one instruction more, and costs the 256 x 256 tile 5 to 20 %, it seems
// where the epilogue no longer stays in the instruction cache from launch to launch: 8192 x 2048 x 8192 with z kept 235 us and 248,
// 8192 x 512 x 2048 30 and 36.)
__device__ __forceinline__ float silu_fast(float z) { return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * z)); }
// float: the exponential as the square of its root
__device__ __forceinline__ float silu(float z) {
    const float root = expf(-0.5f * fabsf(z)), q = 1.0f / fmaf(root, root, 1.0f);
    return z < 0.0f ? (z * root) * (root * q) : z * q;
}

// act(z); act is the same for a whole launch
template <typename T> __device__ __forceinline__ float activate(float z, int act);
template <> __device__ __forceinline__ float activate<bf16_t>(float z, int act) {
    if (act == MOE_ACT_GELU) return gelu_tail_f(z);
    if (act == MOE_ACT_SILU) return silu_fast(z);
    return z;
}
template <> __device__ __forceinline__ float activate<float>(float z, int act) {
    if (act == MOE_ACT_GELU) return z * normal_cdf(z);
    if (act == MOE_ACT_SILU) return silu(z);
    return z;
}

// n values at once: which activation is asked once
template <typename T, int N> __device__ __forceinline__ void activate_all(const float* z, float* y, int act) {
    if (act == MOE_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = activate<T>(z[i], MOE_ACT_GELU);
    } else if (act == MOE_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = activate<T>(z[i], MOE_ACT_SILU);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = z[i];
    }
}

// act'(z) = Phi(z) + z phi(z), or s (1 + z (1 - s)) with s the sigmoid of z.  Exponentials are squares of their roots, which the factors are
// multiplied with one after the other: a slope is a normal number for some way after its exponential has ceased to be one.
template <typename T> __device__ __forceinline__ float activation_slope(float z, int act) {
    constexpr bool FAST = sizeof(T) == 2;
    if (act == MOE_ACT_GELU) {
        float root, cdf;
        if (FAST) cdf = normal_cdf_fast(z, &root);
        else { cdf = normal_cdf(z); root = expf(-0.25f * z * z); }
        return fmaf(z * 0.39894228040143267794f * root, root, cdf);
    }
    if (act == MOE_ACT_SILU) {
        const float root = FAST ? __builtin_amdgcn_exp2f((-0.5f * 1.44269504088896340736f) * fabsf(z)) : expf(-0.5f * fabsf(z)), e = root * root;
        const float q = FAST ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e);
        const float f = fmaf(z, z < 0.0f ? q : e * q, 1.0f);                       // 1 + z (1 - sigmoid(z))
        return z < 0.0f ? (root * f) * (root * q) : q * f;
    }
    return 1.0f;
}

}  // namespace moe
