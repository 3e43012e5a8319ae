// What follows a product in its epilogue: an activation and a residual.  The products' kernels exist with (template flag POST) and without it, so
// that a product alone keeps the registers and instructions that it had.
#pragma once

#include <type_traits>

#include "amq_common.cuh"

namespace amq {

// v Phi(v).  The tail Phi(-|v|) = erfc(|v| / sqrt 2) / 2 by Abramowitz and Stegun's formula 7.1.26 (a polynomial in t = 1 / (1 + p x) times exp(-x^2), within 1.5e-7
// of erf): nothing cancels for v << 0, and a dozen instructions where erfcf takes four times as many (32768 x 1024, 512 vectors: 91 -> 75 us).  Beyond 16 the
// tail is 0 in fp32, and is not multiplied by an infinite v.
__device__ __forceinline__ float gelu(float v)
{
    const float x = 0.70710678f * fabsf(v), t = __fdividef(1.0f, fmaf(0.3275911f, x, 1.0f));
    const float w = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f) * __expf(-x * x);
    return v > 0.0f ? fmaf(-0.5f * fminf(v, 16.0f), w, v) : 0.5f * fmaxf(v, -16.0f) * w;
}

// expf and tanhf rather than faster forms: an activation is a few instructions of a thread that has just folded dozens of integers, and its result is then as near
// to the exact one as the product is.
template <int ACTIVATION> __device__ __forceinline__ float activate(float v)
{
    if (ACTIVATION == AMQ_ACT_RELU) return v < 0.0f ? 0.0f : v;                      // (NaN stays NaN)
    if (ACTIVATION == AMQ_ACT_GELU) return gelu(v);
    if (ACTIVATION == AMQ_ACT_SILU) return __fdividef(fmaxf(v, -1e30f), 1.0f + expf(-v));           // (a denominator beyond 2^126 gives 0, the result's limit)
    if (ACTIVATION == AMQ_ACT_TANH) return tanhf(v);
    if (ACTIVATION == AMQ_ACT_SIGMOID) return __fdividef(1.0f, 1.0f + expf(-v));
    return v;
}

// N values at once: one choice for all of them
template <int N> __device__ __forceinline__ void activate(float (&v)[N], int activation)
{
    auto all = [&](auto kind) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<decltype(kind)::value>(v[i]);
    };
    switch (activation) {
        case AMQ_ACT_RELU: all(std::integral_constant<int, AMQ_ACT_RELU>{}); break;
        case AMQ_ACT_GELU: all(std::integral_constant<int, AMQ_ACT_GELU>{}); break;
        case AMQ_ACT_SILU: all(std::integral_constant<int, AMQ_ACT_SILU>{}); break;
        case AMQ_ACT_TANH: all(std::integral_constant<int, AMQ_ACT_TANH>{}); break;
        case AMQ_ACT_SIGMOID: all(std::integral_constant<int, AMQ_ACT_SIGMOID>{}); break;
        default: break;
    }
}

__device__ __forceinline__ float activate(float v, int activation)
{
    float a[1] = {v};
    activate(a, activation);
    return a[0];
}

}  // namespace amq
