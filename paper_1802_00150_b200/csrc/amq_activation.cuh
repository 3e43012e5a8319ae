// What follows a product in its epilogue: an activation and a residual.  The products' kernels exist with (template flag POST) and without it, so
// that a product alone keeps the registers and instructions that it had.
#pragma once

#include "amq_common.cuh"

namespace amq {

// erfcf, expf and tanhf rather than the fast forms: an activation is a few instructions of a thread that has just folded hundreds of
// products, and its result is then as near to the exact one as the product is.
__device__ __forceinline__ float activate(float v, int activation)
{
    switch (activation) {
        case AMQ_ACT_RELU: return v < 0.0f ? 0.0f : v;                       // (NaN stays NaN)
        case AMQ_ACT_GELU: return 0.5f * v * erfcf(-0.70710678f * v);        // v Phi(v); through erfc, so that nothing cancels for v << 0
        case AMQ_ACT_SILU: return v / (1.0f + expf(-v));
        case AMQ_ACT_TANH: return tanhf(v);
        case AMQ_ACT_SIGMOID: return 1.0f / (1.0f + expf(-v));
        default: return v;
    }
}

}  // namespace amq
