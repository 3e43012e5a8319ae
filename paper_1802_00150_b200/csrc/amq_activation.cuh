// What follows a product in its epilogue: an activation and a residual.  The products' kernels exist with (template flag POST) and without it, so
// that a product alone keeps the registers and instructions that it had.
#pragma once

#include <type_traits>

#include "amq_common.cuh"

namespace amq {

// v Phi(v), from the tail Q(u) = Phi(-u) of u = |v|: v Q(u) for v < 0, where nothing cancels, and v - v Q(u) else.  Q(u) exp(u^2 / 2) is smooth and falls as
// 1 / u, so it is a polynomial in t = 1 / (1 + 0.3 u), with the coefficients whose largest relative error over 0 <= u <= 14 is least (1.5e-7; found by least
// squares whose weights follow the error, Lawson's method).  With the roundings the result is within 1e-6 + 9e-8 v^2 of itself, the second part from the
// exponent's (erfcf is nearer by little, and four times as many instructions: 32768 x 1024, 512 vectors: 91 us).  Beyond 16 the tail is 0 in fp32,
// and is not multiplied by an infinite v.
__device__ __forceinline__ float gelu(float v)
{
    const float u = fabsf(v), t = __fdividef(1.0f, fmaf(0.3f, u, 1.0f));
    float q = 0.035674773f;
    q = fmaf(q, t, -0.15720306f);
    q = fmaf(q, t, 0.20635344f);
    q = fmaf(q, t, -0.053683586f);
    q = fmaf(q, t, 0.1285616f);
    q = fmaf(q, t, 0.0999135f);
    q = fmaf(q, t, 0.12075396f);
    q = fmaf(q, t, 0.1196293f);
    q *= t * __expf(-0.5f * u * u);
    return v > 0.0f ? fmaf(-fminf(v, 16.0f), q, v) : fmaxf(v, -16.0f) * q;
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
