// The batch-1 binary matrix-vector product with an activation and a residual behind it (instantiations of amq_bgemv.cuh; a file of their
// own so that they compile beside the others).
#include "amq_bgemv.cuh"

namespace amq {

amq_status launch_bgemv_post(const GemvParams& p, int k_w, int k_a, cudaStream_t st) { return launch_kw<true>(p, k_w, k_a, st); }

}  // namespace amq
