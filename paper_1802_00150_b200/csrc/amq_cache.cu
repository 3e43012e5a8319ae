// Writing of quantized keys and values into the paged cache (amq_cache.cuh).
#include "amq_cache.cuh"

namespace amq {
namespace {

struct AppendParams {
    CacheView c;
    const uint4* kcodes; const char* kcoeffs; const uint4* vcodes; const char* vcoeffs;         // [batch][count][heads][k][..]
    uint4* to_kcodes; char* to_kcoeffs; uint4* to_vcodes; char* to_vcoeffs;
    int count;
    int chunks, coeffs;                 // pieces of a token: 16 bytes of codes, sizeof(V) of coefficients (of the keys, and as many of the values)
    long long pieces;                   // of all tokens
};

// A thread copies a piece of a token, all of whose heads' rows lie together on both sides.  What it copies is on its way before it knows where to: the chain
// behind that is the length, the table's entry and the store.  (One token of 64 sequences, 8 heads of 128 x 4 bits: 3.3 us, 4.0 with a CTA to a token that
// looks for the place first; 8000 tokens, 20 MB read and written: 6.4 us against 10.7.)  V: of a piece of coefficients.
template <typename V>
__global__ void __launch_bounds__(256)
cache_append_kernel(const __grid_constant__ AppendParams p)
{
    grid_dependency_wait();
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= p.pieces) return;
    const int each = 2 * (p.chunks + p.coeffs);
    const long long token = at / each;
    int piece = (int)(at - token * each);
    const int b = (int)(token / p.count), i = (int)(token - (long long)b * p.count);
    const bool codes = piece < 2 * p.chunks;
    if (!codes) piece -= 2 * p.chunks;
    const int n = codes ? p.chunks : p.coeffs;
    const bool value = piece >= n;
    if (value) piece -= n;
    uint4 chunk;
    V coeff;
    if (codes) chunk = __ldcg((value ? p.vcodes : p.kcodes) + token * n + piece);
    else coeff = __ldcg(reinterpret_cast<const V*>(value ? p.vcoeffs : p.kcoeffs) + token * n + piece);
    const long long t = (long long)p.c.lengths[b] - p.count + i;
    if (t < 0 || t >= (long long)p.c.max_pages * p.c.page_size) return;
    const int slot = slot_of(p.c, b, (int)t);
    if (slot < 0) return;
    if (codes) (value ? p.to_vcodes : p.to_kcodes)[(long long)slot * n + piece] = chunk;
    else reinterpret_cast<V*>(value ? p.to_vcoeffs : p.to_kcoeffs)[(long long)slot * n + piece] = coeff;
}

}  // namespace
}  // namespace amq

extern "C" {

amq_status amq_cache_append(const uint32_t* kcodes, const float* kcoeffs, const uint32_t* vcodes, const float* vcoeffs,
                            uint32_t* cache_kcodes, float* cache_kcoeffs, uint32_t* cache_vcodes, float* cache_vcoeffs,
                            int pages, int page_size, int heads, int d, int k, const int32_t* table, int ld_table, int max_pages,
                            const int32_t* lengths, int batch, int count, void* stream)
{
    amq::AppendParams p{};
    const amq_status s = amq::cache_view(cache_kcodes, cache_kcoeffs, cache_vcodes, cache_vcoeffs, pages, page_size, heads, d, k, table, ld_table, max_pages,
                                         lengths, &p.c);
    if (s != AMQ_OK) return s;
    if (batch < 0 || count < 0) return AMQ_ERR_INVALID_ARG;
    if ((long long)batch * count > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (batch == 0 || count == 0 || max_pages == 0 || pages == 0) return AMQ_OK;       // (no page: every row is left out)
    if (!kcodes || !kcoeffs || !vcodes || !vcoeffs || !table || !lengths || !cache_kcodes || !cache_kcoeffs || !cache_vcodes || !cache_vcoeffs)
        return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(kcodes) || !amq::aligned16(vcodes) || !amq::aligned16(cache_kcodes) || !amq::aligned16(cache_vcodes)) return AMQ_ERR_ALIGNMENT;
    const int rows = heads * k;
    // coefficients four at a time where every token's lie on 16 bytes
    const bool wide = rows % 4 == 0 && amq::aligned16(kcoeffs) && amq::aligned16(vcoeffs) && amq::aligned16(cache_kcoeffs) && amq::aligned16(cache_vcoeffs);
    p.kcodes = reinterpret_cast<const uint4*>(kcodes); p.kcoeffs = reinterpret_cast<const char*>(kcoeffs);
    p.vcodes = reinterpret_cast<const uint4*>(vcodes); p.vcoeffs = reinterpret_cast<const char*>(vcoeffs);
    p.to_kcodes = reinterpret_cast<uint4*>(cache_kcodes); p.to_kcoeffs = reinterpret_cast<char*>(cache_kcoeffs);
    p.to_vcodes = reinterpret_cast<uint4*>(cache_vcodes); p.to_vcoeffs = reinterpret_cast<char*>(cache_vcoeffs);
    p.count = count;
    p.chunks = rows * (p.c.wpr / 4); p.coeffs = wide ? rows / 4 : rows;
    p.pieces = (long long)batch * count * 2 * (p.chunks + p.coeffs);
    const long long grid = (p.pieces + 255) / 256;
    if (grid > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    AMQ_CUDA_TRY(amq::launch_kernel(wide ? amq::cache_append_kernel<float4> : amq::cache_append_kernel<float>, dim3((unsigned)grid), dim3(256), 0,
                                    (cudaStream_t)stream, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // extern "C"
