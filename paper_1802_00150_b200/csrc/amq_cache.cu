// A paged cache that holds keys and values in packed planes, as the row quantizer leaves them: writing of new rows, and attention over it.
//
//   s[t] = scale * sum_i a[t][i] (q . b[t][i]),   p = softmax over the visible t,   o = sum_t p[t] sum_i a'[t][i] b'[t][i]
// with the planes b, b' (+-1) and coefficients a, a' of token t's key and value.
#include "amq_common.cuh"

namespace amq {
namespace {

struct CacheView {
    const uint32_t* kcodes; const float* kcoeffs; const uint32_t* vcodes; const float* vcoeffs;
    int pages, page_size, heads, d, k, wpr;
    const int32_t* table; int ld_table, max_pages;
    const int32_t* lengths;
};

__device__ __forceinline__ int visible_length(const CacheView& c, int b)
{
    const long long most = (long long)c.max_pages * c.page_size;
    const int n = c.lengths[b];
    return n < 0 ? 0 : n < most ? n : (int)most;
}

// slot (token position in the whole cache) of token t of sequence b, -1 where the table names no page
__device__ __forceinline__ long long slot_of(const CacheView& c, int b, int t)
{
    const int page = c.table[(size_t)b * c.ld_table + t / c.page_size];
    return page >= 0 && page < c.pages ? (long long)page * c.page_size + t % c.page_size : -1;
}

struct AppendParams {
    CacheView c;
    const uint4* kcodes; const float* kcoeffs; const uint4* vcodes; const float* vcoeffs;       // [batch][count][heads][k][..]
    uint4* to_kcodes; float* to_kcoeffs; uint4* to_vcodes; float* to_vcoeffs;
    int count;
};

// one CTA per new token: its rows of all heads are contiguous on both sides
__global__ void __launch_bounds__(128)
cache_append_kernel(const __grid_constant__ AppendParams p)
{
    grid_dependency_wait();
    const int b = blockIdx.x / p.count, i = blockIdx.x % p.count;
    const int t = p.c.lengths[b] - p.count + i;
    if (t < 0 || t >= (long long)p.c.max_pages * p.c.page_size) return;
    const long long slot = slot_of(p.c, b, t);
    if (slot < 0) return;
    const int rows = p.c.heads * p.c.k, chunks = rows * (p.c.wpr / 4);
    const size_t from = blockIdx.x, to = (size_t)slot;
    for (int j = threadIdx.x; j < chunks; j += 128) {
        p.to_kcodes[to * chunks + j] = p.kcodes[from * chunks + j];
        p.to_vcodes[to * chunks + j] = p.vcodes[from * chunks + j];
    }
    for (int j = threadIdx.x; j < rows; j += 128) {
        p.to_kcoeffs[to * rows + j] = p.kcoeffs[from * rows + j];
        p.to_vcoeffs[to * rows + j] = p.vcoeffs[from * rows + j];
    }
}

struct AttentionParams {
    CacheView c;
    const float* q; long long q_batch, q_token, q_head;
    int q_len, q_heads, group;
    float scale;
    float* out;
};

constexpr int DPL = AMQ_MAX_HEAD_DIM / 32;      // dimensions of a lane

// one CTA per query row; its warps take every fourth token
__global__ void __launch_bounds__(128)
cache_attention_kernel(const __grid_constant__ AttentionParams p)
{
    __shared__ float s_m[4], s_l[4], s_o[4][AMQ_MAX_HEAD_DIM];
    grid_dependency_wait();
    const CacheView& c = p.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int h = blockIdx.x % p.q_heads, i = blockIdx.x / p.q_heads % p.q_len, b = blockIdx.x / p.q_heads / p.q_len, kv = h / p.group;
    const int seen = visible_length(c, b) - p.q_len + 1 + i;
    const float* q = p.q + b * p.q_batch + i * p.q_token + h * p.q_head;
    float qv[DPL], o[DPL];
#pragma unroll
    for (int j = 0; j < DPL; ++j) { qv[j] = lane + 32 * j < c.d ? q[lane + 32 * j] : 0.0f; o[j] = 0.0f; }
    float m = -INFINITY, l = 0.0f;
    for (int t = warp; t < seen; t += 4) {
        const long long slot = slot_of(c, b, t);
        if (slot < 0) continue;
        const size_t row = ((size_t)slot * c.heads + kv) * c.k;
        float s = 0.0f;
        for (int pl = 0; pl < c.k; ++pl) {
            float dot = 0.0f;
#pragma unroll
            for (int j = 0; j < DPL; ++j) dot += (c.kcodes[(row + pl) * c.wpr + j] >> lane & 1) ? qv[j] : -qv[j];
            s += c.kcoeffs[row + pl] * dot;
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= p.scale;
        const float m_new = fmaxf(m, s), corr = expf(m - m_new), w = expf(s - m_new);
        l = l * corr + w;
#pragma unroll
        for (int j = 0; j < DPL; ++j) o[j] *= corr;
        for (int pl = 0; pl < c.k; ++pl) {
            const float a = w * c.vcoeffs[row + pl];
#pragma unroll
            for (int j = 0; j < DPL; ++j) o[j] += (c.vcodes[(row + pl) * c.wpr + j] >> lane & 1) ? a : -a;
        }
        m = m_new;
    }
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
    for (int j = 0; j < DPL; ++j) s_o[warp][lane + 32 * j] = o[j];
    __syncthreads();
    const float M = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float total = 0.0f, sum = 0.0f;
    for (int w = 0; w < 4; ++w) {
        const float f = s_l[w] == 0.0f ? 0.0f : expf(s_m[w] - M);
        total += s_l[w] * f;
        sum += s_o[w][threadIdx.x] * f;
    }
    if (threadIdx.x < c.d) p.out[(size_t)blockIdx.x * c.d + threadIdx.x] = total == 0.0f ? 0.0f : sum / total;
}

amq_status cache_view(const uint32_t* kcodes, const float* kcoeffs, const uint32_t* vcodes, const float* vcoeffs, int pages, int page_size, int heads,
                      int d, int k, const int32_t* table, int ld_table, int max_pages, const int32_t* lengths, CacheView* out)
{
    if (pages < 0 || page_size < 1 || heads < 1 || d < 1 || max_pages < 0 || ld_table < max_pages) return AMQ_ERR_INVALID_ARG;
    if (!valid_k(k) || d > AMQ_MAX_HEAD_DIM || heads > 65535) return AMQ_ERR_UNSUPPORTED;
    if ((long long)max_pages * page_size > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    *out = {kcodes, kcoeffs, vcodes, vcoeffs, pages, page_size, heads, d, k, words_per_row(d), table, ld_table, max_pages, lengths};
    return AMQ_OK;
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
    if (batch == 0 || count == 0 || max_pages == 0) return AMQ_OK;
    if (!kcodes || !kcoeffs || !vcodes || !vcoeffs || !table || !lengths || !cache_kcodes || !cache_kcoeffs || !cache_vcodes || !cache_vcoeffs)
        return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(kcodes) || !amq::aligned16(vcodes) || !amq::aligned16(cache_kcodes) || !amq::aligned16(cache_vcodes)) return AMQ_ERR_ALIGNMENT;
    p.kcodes = reinterpret_cast<const uint4*>(kcodes); p.kcoeffs = kcoeffs; p.vcodes = reinterpret_cast<const uint4*>(vcodes); p.vcoeffs = vcoeffs;
    p.to_kcodes = reinterpret_cast<uint4*>(cache_kcodes); p.to_kcoeffs = cache_kcoeffs;
    p.to_vcodes = reinterpret_cast<uint4*>(cache_vcodes); p.to_vcoeffs = cache_vcoeffs;
    p.count = count;
    AMQ_CUDA_TRY(amq::launch_kernel(amq::cache_append_kernel, dim3((unsigned)(batch * count)), dim3(128), 0, (cudaStream_t)stream, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

size_t amq_cache_attention_workspace_bytes(int batch, int q_len, int q_heads, int heads, int d, int max_tokens)
{
    return 0;
}

amq_status amq_cache_attention(const float* q, long long q_batch, long long q_token, long long q_head,
                               const uint32_t* cache_kcodes, const float* cache_kcoeffs, const uint32_t* cache_vcodes, const float* cache_vcoeffs,
                               int pages, int page_size, int heads, int d, int k, const int32_t* table, int ld_table, int max_pages,
                               const int32_t* lengths, int batch, int q_len, int q_heads, float scale, float* out,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    amq::AttentionParams p{};
    const amq_status s = amq::cache_view(cache_kcodes, cache_kcoeffs, cache_vcodes, cache_vcoeffs, pages, page_size, heads, d, k, table, ld_table, max_pages,
                                         lengths, &p.c);
    if (s != AMQ_OK) return s;
    if (batch < 0 || q_len < 0 || q_heads < 1 || q_heads % heads) return AMQ_ERR_INVALID_ARG;
    if ((long long)batch * q_len * q_heads > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (batch == 0 || q_len == 0) return AMQ_OK;
    if (!q || !out || !lengths || (max_pages > 0 && !table)) return AMQ_ERR_INVALID_ARG;
    if (pages > 0 && (!cache_kcodes || !cache_kcoeffs || !cache_vcodes || !cache_vcoeffs)) return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(cache_kcodes) || !amq::aligned16(cache_vcodes)) return AMQ_ERR_ALIGNMENT;
    p.q = q; p.q_batch = q_batch; p.q_token = q_token; p.q_head = q_head;
    p.q_len = q_len; p.q_heads = q_heads; p.group = q_heads / heads; p.scale = scale; p.out = out;
    AMQ_CUDA_TRY(amq::launch_kernel(amq::cache_attention_kernel, dim3((unsigned)(batch * q_len * q_heads)), dim3(128), 0, (cudaStream_t)stream, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // extern "C"
