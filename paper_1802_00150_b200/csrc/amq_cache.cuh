// A paged cache of keys and values in packed planes, as the kernels of its calls see it.
#pragma once

#include "amq_common.cuh"

namespace amq {

struct CacheView {
    const uint32_t* kcodes; const float* kcoeffs; const uint32_t* vcodes; const float* vcoeffs;
    int pages, page_size, page_shift, heads, d, k, wpr;     // page_shift: of a page size that is a power of two, else -1
    const int32_t* table; int ld_table, max_pages;
    const int32_t* lengths;
};

__device__ __forceinline__ int visible_length(const CacheView& c, int b)
{
    const long long most = (long long)c.max_pages * c.page_size;
    const int n = c.lengths[b];
    return n < 0 ? 0 : n < most ? n : (int)most;
}

// place of a token's page in a row of the table
__device__ __forceinline__ int page_index(const CacheView& c, int t) { return c.page_shift >= 0 ? t >> c.page_shift : t / c.page_size; }

// slot (token position in the whole cache) of token t on a page, -1 where that is none
__device__ __forceinline__ int slot_on(const CacheView& c, int page, int t)
{
    return page >= 0 && page < c.pages ? page * c.page_size + (t - page_index(c, t) * c.page_size) : -1;
}

// the same for token t of sequence b
__device__ __forceinline__ int slot_of(const CacheView& c, int b, int t)
{
    return slot_on(c, c.table[(size_t)b * c.ld_table + page_index(c, t)], t);
}

// arguments that the calls share, checked
inline amq_status cache_view(const uint32_t* kcodes, const float* kcoeffs, const uint32_t* vcodes, const float* vcoeffs, int pages, int page_size, int heads,
                      int d, int k, const int32_t* table, int ld_table, int max_pages, const int32_t* lengths, CacheView* out)
{
    if (pages < 0 || page_size < 1 || heads < 1 || d < 1 || max_pages < 0 || ld_table < max_pages) return AMQ_ERR_INVALID_ARG;
    if (!valid_k(k) || d > AMQ_MAX_HEAD_DIM || heads > 65535) return AMQ_ERR_UNSUPPORTED;
    if ((long long)max_pages * page_size > AMQ_MAX_TOKENS || (long long)pages * page_size > AMQ_MAX_TOKENS) return AMQ_ERR_UNSUPPORTED;
    int shift = -1;
    for (int i = 0; i < 31; ++i) if (page_size == 1 << i) shift = i;
    *out = {kcodes, kcoeffs, vcodes, vcoeffs, pages, page_size, shift, heads, d, k, words_per_row(d), table, ld_table, max_pages, lengths};
    return AMQ_OK;
}

}  // namespace amq
