// Entry points of the batch-1 binary matrix-vector product (amq_bgemv.cuh).
#include "amq_bgemv.cuh"

namespace amq {

// the form with an activation or a residual behind the product: the same kernel, instantiated in amq_bgemv_post.cu
amq_status launch_bgemv_post(const GemvParams& p, int k_w, int k_a, cudaStream_t st);

bool gemv_supported(const GemmArgs& a)
{
    return a.batch == 1 && (a.epilogue == EPI_Y || a.epilogue == EPI_DOTS) && words_per_row(a.n) / 4 <= 64;
}

amq_status launch_binary_gemv(const GemmArgs& a, cudaStream_t st)
{
    if (!gemv_supported(a)) return AMQ_ERR_UNSUPPORTED;
    GemvParams p;
    p.W = reinterpret_cast<const uint4*>(a.Wcodes);
    p.Walpha = a.Walpha;
    p.x = reinterpret_cast<const uint4*>(a.xcodes);
    p.xbeta = a.xbeta;
    p.bias = a.bias;
    p.y = a.y;
    p.D = a.D;
    p.m = a.m; p.n = a.n; p.CH = words_per_row(a.n) / 4;
    p.epilogue = a.epilogue;
    p.overlap = a.overlap_with_previous || (a.post && a.from_entry);    // (the kernel waits before it reads anything)
    p.xf = nullptr; p.T = 0; p.xcodes_out = nullptr; p.xbeta_out = nullptr;
    p.activation = a.activation; p.residual = a.residual;
    return a.post ? launch_bgemv_post(p, a.k_w, a.k_a, st) : launch_kw<false>(p, a.k_w, a.k_a, st);
}

bool quantized_gemv_supported(int n) { return n >= 1 && words_per_row(n) / 4 <= FQ_MAX_CH; }

amq_status launch_quantized_gemv(const uint32_t* Wcodes, const float* Walpha, int m, int n, int k_w, const float* x, int k_a, int T,
                                 const float* bias, float* y, uint32_t* xcodes_out, float* xbeta_out, cudaStream_t st,
                                 bool overlap_with_previous)
{
    if (!quantized_gemv_supported(n)) return AMQ_ERR_UNSUPPORTED;
    GemvParams p;
    p.W = reinterpret_cast<const uint4*>(Wcodes);
    p.Walpha = Walpha;
    p.x = nullptr; p.xbeta = nullptr;
    p.bias = bias;
    p.y = y; p.D = nullptr;
    p.m = m; p.n = n; p.CH = words_per_row(n) / 4;
    p.epilogue = EPI_Y;
    p.overlap = overlap_with_previous;
    p.xf = x; p.T = T; p.xcodes_out = xcodes_out; p.xbeta_out = xbeta_out;
    p.activation = 0; p.residual = nullptr;
    return launch_kw<false>(p, k_w, k_a, st);
}

}  // namespace amq

extern "C" amq_status amq_quantized_gemv(const uint32_t* Wcodes, const float* Walpha, int m, int n, int k_w,
                                         const float* x, int k_a, int T, const float* bias, float* y,
                                         uint32_t* xcodes_out, float* xbeta_out, void* stream)
{
    if (m < 0 || n < 1) return AMQ_ERR_INVALID_ARG;
    if (!amq::valid_k(k_w) || !amq::valid_k(k_a) || T < 0 || !amq::quantized_gemv_supported(n)) return AMQ_ERR_UNSUPPORTED;
    if (m == 0) return AMQ_OK;
    if (!Wcodes || !Walpha || !x || !y) return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(Wcodes) || (xcodes_out && !amq::aligned16(xcodes_out))) return AMQ_ERR_ALIGNMENT;
    return amq::launch_quantized_gemv(Wcodes, Walpha, m, n, k_w, x, k_a, T, bias, y, xcodes_out, xbeta_out,
                                      (cudaStream_t)stream, false);
}
