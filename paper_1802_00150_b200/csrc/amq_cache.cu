// A paged cache that holds keys and values in packed planes, as the row quantizer leaves them: writing of new rows, and attention over it.
//
//   s[t] = scale * sum_i a[t][i] (q . b[t][i]),   p = softmax over the visible t,   o = sum_t p[t] sum_i a'[t][i] b'[t][i]
// with the planes b, b' (+-1) and coefficients a, a' of token t's key and value.
#include <stddef.h>

#include "amq_common.cuh"
#include "amq_pairs.cuh"

namespace amq {
namespace {

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

// slot (token position in the whole cache) of token t of sequence b, -1 where the table names no page
__device__ __forceinline__ int slot_of(const CacheView& c, int b, int t)
{
    const int j = c.page_shift >= 0 ? t >> c.page_shift : t / c.page_size;
    const int page = c.table[(size_t)b * c.ld_table + j];
    return page >= 0 && page < c.pages ? page * c.page_size + (t - j * c.page_size) : -1;
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
    const int slot = slot_of(p.c, b, t);
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
    int rows, row_blocks;               // query rows of a key head: q_len * group, in blocks of ROWS
    int splits;                         // shares of a sequence's tokens
    bool wide;                          // coefficient rows on their own size (4, 8 or 16 bytes)
    float scale;
    float* out;
    float* part; float2* part_ml;       // splits > 1: unnormalised results and {maximum, sum} of each share, [row][split]
};

constexpr int WARPS = 4;
constexpr int TILE = 32;                // tokens
#ifndef AT_STAGES
#define AT_STAGES 3
#endif
#ifndef AT_MINB
#define AT_MINB 3
#endif
constexpr int STAGES = AT_STAGES;
constexpr int ROWS = 4;                 // query rows of a CTA
constexpr float MAGIC = 12582912.0f;    // 1.5 2^23: a float of this size holds an integer of 22 bits in its low bits
constexpr int MAGIC_BITS = 0x4B400000;

// chunks (16 bytes: a plane of up to 128 bits) and coefficients of a token in shared memory; four for three
__host__ __device__ constexpr int pitch(int k) { return k == 3 ? 4 : k; }
template <int K> struct Stage {
    uint4 k[TILE * pitch(K)], v[TILE * pitch(K)];
    float ka[TILE * pitch(K)], va[TILE * pitch(K)];
};
// a tile's coefficients by planes
template <int K> struct Coefficients { float k[K][TILE], v[K][TILE]; };
// place of a token's plane: spread so that neither access pattern below meets a bank twice
template <int K> __device__ __forceinline__ int place(int token, int plane)
{
    if (pitch(K) == 4) return token * 4 + (plane ^ (token >> 1 & 3));
    if (pitch(K) == 2) return token * 2 + (plane ^ (token >> 2 & 1));
    return token;
}

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void* from, bool real)
{
    const int n = real ? BYTES : 0;                 // (nothing is read for the others: zeros are written)
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(from), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" :: "r"(dst), "l"(from), "r"(n), "n"(BYTES) : "memory");
}

// a token's coefficients from shared memory, at once
template <int K> __device__ __forceinline__ void load_row(const float* from, float (&v)[K])
{
    if constexpr (K == 4) { const float4 a = *reinterpret_cast<const float4*>(from); v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
    else if constexpr (K == 2) { const float2 a = *reinterpret_cast<const float2*>(from); v[0] = a.x; v[1] = a.y; }
    else
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] = from[i];
}

__device__ __forceinline__ void mma_s8u8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// the first of a chain: the sum starts from `start`, whose registers stay (a constant in place would be moved there each time)
__device__ __forceinline__ void mma_s8u8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const int (&start)[4])
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(start[0]), "r"(start[1]), "r"(start[2]), "r"(start[3]));
}

// two sums as floats: integers of up to 22 bits on top of MAGIC
__device__ __forceinline__ f32x2 sums2(int a, int b) { return add2(pack2(__int_as_float(a), __int_as_float(b)), pack2(-MAGIC, -MAGIC)); }

__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

// The products run on the integer tensor cores, on the planes' bits as they are stored: a word ANDed with 0x01010101 << j is four bytes of 0 or
// 2^j, an operand of mma.m16n8k32 with the query (or the weights) as digits of eight bits.  A query row is four rows of the operand, its
// digits, so that four query rows fill the 16 rows of an instruction, and the product is exact:
//   q = sum_digits 256^i d_i (31-bit fixed point; elements whose bits lie at position j of a byte are held divided by 2^j),
//   q . b = 2 sum_{bit = 1} q - sum q.
// Nothing else in this kernel is near the tensor cores' or the memory's pace: per 8 tokens of 4 bits 64 AND, 33 MMAs, 1280 bytes.
//
// A warp takes tiles of 32 tokens on its own (its copies, through a ring of its own stages; the softmax's running maximum and sum; partial sums), the
// CTA's four warps are joined at the end, and shares of a sequence (`splits`) by a second kernel.
//
// Lane l = 4 g + c of an MMA holds rows g and g + 8: digits g / 4 and 2 + g / 4 of query row g mod 4.  For keys, column g is token g of eight and c the
// word of the plane; results are those of tokens 2 c, 2 c + 1.  For values, c stands for the same two tokens, so weights never change
// lanes, and column g for dimensions 16 g .. 16 g + 15, one per MMA.
template <int K>
__global__ void __launch_bounds__(WARPS * 32, AT_MINB)
cache_attention_kernel(const __grid_constant__ AttentionParams p)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float s_m[WARPS][ROWS], s_l[WARPS][ROWS];
    __shared__ uint32_t s_largest[WARPS][ROWS];
    __shared__ uint4 s_digits[WARPS][32];
    __shared__ int s_sum[WARPS][8][2];
    const CacheView& cv = p.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3, r = g & 3;
    const bool upper = g < 4;           // rows g, g + 8: digits 3 and 1, else 2 and 0
    const uint32_t digit0 = upper ? 0x73u : 0x62u, digit1 = upper ? 0x51u : 0x40u;      // these bytes of two words
    Stage<K>* stages = reinterpret_cast<Stage<K>*>(smem_raw) + warp * STAGES;
    const uint32_t stage_at = (uint32_t)__cvta_generic_to_shared(stages);
    Coefficients<K>& coef = (reinterpret_cast<Coefficients<K>*>(reinterpret_cast<Stage<K>*>(smem_raw) + WARPS * STAGES))[warp];

    int at = blockIdx.x;
    const int rb = at % p.row_blocks; at /= p.row_blocks;
    const int kv = at % cv.heads; at /= cv.heads;
    const int split = at % p.splits, b = at / p.splits;

    grid_dependency_wait();
    const int length = visible_length(cv, b);
    const int last_row = min(rb * ROWS + ROWS, p.rows) - 1;
    const int limit = max(length - p.q_len + 1 + last_row / p.group, 0);        // of the block's last row: no other sees more
    const int row = rb * ROWS + r;
    const int my_limit = row < p.rows ? length - p.q_len + 1 + row / p.group : limit;
    const int tiles = limit > 0 ? (limit - 1) / TILE + 1 : 0;
    const int tile0 = (int)((long long)tiles * split / p.splits), tile1 = (int)((long long)tiles * (split + 1) / p.splits);

    auto slot_at = [&](int tile) {
        const int t = tile * TILE + lane;
        return tile < tile1 && t < limit ? slot_of(cv, b, t) : -1;
    };
    // planes: K lanes a token, so that an instruction's lanes meet few lines; coefficients: a lane a token
    const uint32_t step = (uint32_t)cv.heads * K;           // planes of a token (at most 2^18)
    const char* const kcodes = reinterpret_cast<const char*>(cv.kcodes) + (size_t)kv * K * 16;
    const char* const vcodes = reinterpret_cast<const char*>(cv.vcodes) + (size_t)kv * K * 16;
    const char* const kcoeffs = reinterpret_cast<const char*>(cv.kcoeffs + (size_t)kv * K);
    const char* const vcoeffs = reinterpret_cast<const char*>(cv.vcoeffs + (size_t)kv * K);
    auto issue = [&](uint32_t st, int slot) {               // st: address of the stage
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int idx = i * 32 + lane, token = idx / K, plane = idx % K;
            const int s = __shfl_sync(0xffffffffu, slot, token);
            const uint64_t from = (uint64_t)(uint32_t)max(s, 0) * (step * 16u);
            const uint32_t to = st + place<K>(token, plane) * 16;
            copy_async<16>(to, kcodes + plane * 16 + from, s >= 0);
            copy_async<16>(to + (uint32_t)offsetof(Stage<K>, v), vcodes + plane * 16 + from, s >= 0);
        }
        const uint64_t from = (uint64_t)(uint32_t)max(slot, 0) * (step * 4u);
        const uint32_t ka = st + (uint32_t)offsetof(Stage<K>, ka) + lane * pitch(K) * 4, va = st + (uint32_t)offsetof(Stage<K>, va) + lane * pitch(K) * 4;
        constexpr int UNIT = K == 3 ? 1 : K;
        if (p.wide) {
#pragma unroll
            for (int i = 0; i < K; i += UNIT) {
                copy_async<4 * UNIT>(ka + 4 * i, kcoeffs + 4 * i + from, slot >= 0);
                copy_async<4 * UNIT>(va + 4 * i, vcoeffs + 4 * i + from, slot >= 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i) {
                copy_async<4>(ka + 4 * i, kcoeffs + 4 * i + from, slot >= 0);
                copy_async<4>(va + 4 * i, vcoeffs + 4 * i + from, slot >= 0);
            }
        }
    };
    auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };

    int tile = tile0 + warp;
    uint32_t real[STAGES];              // tokens on a page, per stage
    int slot = slot_at(tile);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        const int now = slot;
        slot = slot_at(tile + (s + 1) * WARPS);
        real[s] = __ballot_sync(0xffffffffu, now >= 0);
        if (real[s]) issue(stage_at + s * (uint32_t)sizeof(Stage<K>), now);
        commit();
    }

    // The query's digits as the MMAs take them, and the digits' sums (times the bytes' weights) over the row.  A warp makes those of two bit positions.
    uint32_t aq[4][4];
    float half_sum[2], factor;
    {
        float x[8];
        uint32_t largest = 0;
        const int i = row / p.group, h = kv * p.group + row % p.group, first = 32 * c + 2 * warp;
        const float* q = p.q + b * p.q_batch + i * p.q_token + h * p.q_head + first;
#pragma unroll
        for (int byte = 0; byte < 4; ++byte)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                x[2 * byte + j] = row < p.rows && first + 8 * byte + j < cv.d ? q[8 * byte + j] : 0.0f;
                largest = max(largest, __float_as_uint(x[2 * byte + j]) & 0x7fffffffu);
            }
        largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
        largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
        if (upper && c == 0) s_largest[warp][r] = largest;
        __syncthreads();
        largest = max(max(s_largest[0][r], s_largest[1][r]), max(s_largest[2][r], s_largest[3][r]));
        const int e = max((int)(largest >> 23), 29);
        const bool finite = largest < 0x7f800000u;
        const float to_fixed = finite ? __int_as_float((283 - e) << 23) : 0.0f;         // largest element below 2^30
        const float to_fixed_here = to_fixed * __int_as_float((127 - 2 * warp) << 23);
        int sum[2] = {0, 0};
        uint32_t a[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t y[4];
#pragma unroll
            for (int byte = 0; byte < 4; ++byte) {
                y[byte] = (uint32_t)__float2int_rn(x[2 * byte + j] * to_fixed_here * (j ? 0.5f : 1.0f)) + 0x80808080u;
#pragma unroll
                for (int w = 0; w < 2; ++w) sum[w] += ((int)(__byte_perm(y[byte], 0, w ? digit1 & 0x7u : digit0 & 0x7u) & 255u) - 128) * (1 << j);
            }
            a[2 * j] = __byte_perm(__byte_perm(y[0], y[1], digit0), __byte_perm(y[2], y[3], digit0), 0x5410) ^ 0x80808080u;
            a[2 * j + 1] = __byte_perm(__byte_perm(y[0], y[1], digit1), __byte_perm(y[2], y[3], digit1), 0x5410) ^ 0x80808080u;
        }
        s_digits[warp][lane] = make_uint4(a[0], a[1], a[2], a[3]);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 1);
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 2);
            if (c == 0) s_sum[warp][g][w] = sum[w] * (1 << (2 * warp));
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 d = s_digits[j][lane];
            aq[j][0] = d.x; aq[j][1] = d.y; aq[j][2] = d.z; aq[j][3] = d.w;
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) half_sum[w] = 0.5f * (float)(s_sum[0][g][w] + s_sum[1][g][w] + s_sum[2][g][w] + s_sum[3][g][w]);
        factor = finite ? 1.0f / to_fixed * p.scale * (2.0f * 1.44269504f) : NAN;       // scores in units of log 2
    }
    const float w0 = upper ? 16777216.0f : 65536.0f, w1 = upper ? 256.0f : 1.0f;        // the digits' weights
    const f32x2 w0_2 = pack2(w0, w0), w1_2 = pack2(w1, w1);
    const f32x2 minus_half0 = pack2(-half_sum[0], -half_sum[0]), minus_half1 = pack2(-half_sum[1], -half_sum[1]);
    const uint32_t half = g & 1 ? 0x7362u : 0x5140u;        // bytes of the plane words that hold dimensions 16 g ..
    int start[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("mov.b32 %0, %1;" : "=r"(start[i]) : "n"(MAGIC_BITS));

    float m = -INFINITY, l = 0.0f;
    f32x2 o[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] = pack2(0.0f, 0.0f);

    // this lane's words of a plane: of token g of eight (keys), of token 2 c (values; the next token's lie a pitch on)
    uint32_t kat[K], vat[K];
#pragma unroll
    for (int i = 0; i < K; ++i) {
        kat[i] = place<K>(g, i) * 16 + c * 4;
        vat[i] = (uint32_t)offsetof(Stage<K>, v) + place<K>(2 * c, i) * 16 + (g >> 1) * 4;
    }
    int stage = 0;
    for (; tile < tile1; tile += WARPS) {
        {
            const int now = slot;
            slot = slot_at(tile + STAGES * WARPS);
            real[STAGES - 1] = __ballot_sync(0xffffffffu, now >= 0);
            __syncwarp();
            if (real[STAGES - 1]) issue(stage_at + (stage == 0 ? STAGES - 1 : stage - 1) * (uint32_t)sizeof(Stage<K>), now);
            commit();
            asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 1) : "memory");
            __syncwarp();
        }
        const Stage<K>& st = stages[stage];
        const char* const words = reinterpret_cast<const char*>(&st);
        const uint32_t on_a_page = real[0];
#pragma unroll
        for (int q = 0; q < STAGES - 1; ++q) real[q] = real[q + 1];
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (on_a_page == 0) continue;           // (nothing was copied)
        // tokens that this lane's row sees
        const int left = my_limit - tile * TILE;
        const uint32_t seen = on_a_page & (left >= TILE ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u);

        // The coefficients by planes, so that those of tokens 2 c, 2 c + 1 lie together; the values' largest decides the fixed point of the tile's
        // weights.  (The barrier behind the copies lies behind everybody's reading of the last tile's.)
        uint32_t largest = 0;
        float va[K];
        float ka[K];
        load_row<K>(st.ka + lane * pitch(K), ka);
        load_row<K>(st.va + lane * pitch(K), va);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            coef.k[i][lane] = ka[i];
            largest = max(largest, __float_as_uint(va[i]) & 0x7fffffffu);
        }
        largest = __reduce_max_sync(0xffffffffu, largest);
        if (largest >= 0x7f800000u) {           // NaN or infinite coefficients: they count for the rows that see them, and for those only
            bool bad = false;
            largest = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                if (!isfinite(va[i])) { bad = true; va[i] = 0.0f; }
                largest = max(largest, __float_as_uint(va[i]) & 0x7fffffffu);
            }
            largest = __reduce_max_sync(0xffffffffu, largest);
            if (__ballot_sync(0xffffffffu, bad) & seen) l = NAN;
        }
#pragma unroll
        for (int i = 0; i < K; ++i) coef.v[i][lane] = va[i];
        __syncwarp();
        const int ev = max((int)(largest >> 23), 30);
        const float to_fixed = __int_as_float((283 - ev) << 23), from_fixed = __int_as_float((ev - 29) << 23);       // products below 2^30

        // scores of tokens 8 n + 2 c, 8 n + 2 c + 1
        float s[4][2];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            f32x2 x = 0, y = 0, all = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                int acc[4];
                const uint32_t w = *reinterpret_cast<const uint32_t*>(words + kat[i] + n * 8 * pitch(K) * 16);
                mma_s8u8(acc, aq[0], w & 0x01010101u, w & 0x02020202u, start);
#pragma unroll
                for (int j = 1; j < 4; ++j) mma_s8u8(acc, aq[j], w & (0x01010101u << (2 * j)), w & (0x02020202u << (2 * j)));
                const f32x2 a = *reinterpret_cast<const f32x2*>(&coef.k[i][8 * n + 2 * c]);
                x = i ? fma2(a, sums2(acc[0], acc[1]), x) : mul2(a, sums2(acc[0], acc[1]));
                y = i ? fma2(a, sums2(acc[2], acc[3]), y) : mul2(a, sums2(acc[2], acc[3]));
                all = i ? add2(all, a) : a;
            }
            x = fma2(minus_half0, all, x);
            y = fma2(minus_half1, all, y);
            unpack2(fma2(w0_2, x, mul2(w1_2, y)), s[n][0], s[n][1]);
#pragma unroll
            for (int e = 0; e < 2; ++e) s[n][e] = (s[n][e] + __shfl_xor_sync(0xffffffffu, s[n][e], 16)) * factor;
        }
        if (__any_sync(0xffffffffu, seen != 0xffffffffu)) {
            const uint32_t mine = seen >> (2 * c);
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) s[n][e] = mine >> (8 * n + e) & 1 ? s[n][e] : -INFINITY;
        }
        // weights, relative to the tile's maximum
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(s[n][0], s[n][1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float ref = top == -INFINITY ? 0.0f : top, m_new = fmaxf(m, top), m_ref = m_new == -INFINITY ? 0.0f : m_new;
        const float corr = exp2_approx(m - m_ref), tile_factor = exp2_approx(top - m_ref);
        m = m_new;
        float sum = 0.0f;
        // weights times coefficients as digits: an MMA's 32 positions are 32 / pitch tokens, 8 / pitch of them this lane's
        constexpr int PK = pitch(K);            // MMA steps of a tile
        uint32_t ap[PK][4], bv[PK][2][2];
        uint32_t y[8][PK], word[8][PK];         // by this lane's tokens, (n, e) = (0, 0), (0, 1), (1, 0), ..
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const float e0 = exp2_approx(s[n][0] - ref), e1 = exp2_approx(s[n][1] - ref);
            sum += e0 + e1;
            const f32x2 ws = mul2(pack2(e0, e1), pack2(to_fixed, to_fixed));
#pragma unroll
            for (int i = 0; i < PK; ++i) {
                if (i >= K) { y[2 * n][i] = y[2 * n + 1][i] = 0x80808080u; word[2 * n][i] = word[2 * n + 1][i] = 0u; continue; }
                const int j = i < K ? i : 0;
                float f0, f1;
                unpack2(mul2(ws, *reinterpret_cast<const f32x2*>(&coef.v[j][8 * n + 2 * c])), f0, f1);
                y[2 * n][i] = (uint32_t)__float2int_rn(f0) + 0x80808080u;
                y[2 * n + 1][i] = (uint32_t)__float2int_rn(f1) + 0x80808080u;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    word[2 * n + e][i] = *reinterpret_cast<const uint32_t*>(words + vat[j] + (n * 8 + e) * pitch(K) * 16);
            }
        }
#pragma unroll
        for (int z = 0; z < PK; ++z)
#pragma unroll
            for (int side = 0; side < 2; ++side) {
                uint32_t yy[4], ww[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    yy[u] = y[(2 * z + side) * (4 / PK) + u / PK][u % PK];
                    ww[u] = word[(2 * z + side) * (4 / PK) + u / PK][u % PK];
                }
                ap[z][2 * side] = __byte_perm(__byte_perm(yy[0], yy[1], digit0), __byte_perm(yy[2], yy[3], digit0), 0x5410) ^ 0x80808080u;
                ap[z][2 * side + 1] = __byte_perm(__byte_perm(yy[0], yy[1], digit1), __byte_perm(yy[2], yy[3], digit1), 0x5410) ^ 0x80808080u;
                const uint32_t t0 = __byte_perm(ww[0], ww[1], half), t1 = __byte_perm(ww[2], ww[3], half);
                bv[z][side][0] = __byte_perm(t0, t1, 0x5410);
                bv[z][side][1] = __byte_perm(t0, t1, 0x7632);
            }
        l = fmaf(l, corr, sum * tile_factor);
        int ones[4];
        mma_s8u8(ones, ap[0], 0x01010101u, 0x01010101u, start);
#pragma unroll
        for (int z = 1; z < PK; ++z) mma_s8u8(ones, ap[z], 0x01010101u, 0x01010101u);
        const float unit = tile_factor * from_fixed * w1;           // (w0 = 2^16 w1)
        const float base = -unit * fmaf(65536.0f, __int_as_float(ones[0]) - MAGIC, __int_as_float(ones[2]) - MAGIC);
        const f32x2 base_2 = pack2(base, base), corr_2 = pack2(corr, corr);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const f32x2 f = pack2(unit * (2.0f / (1 << j)), unit * (2.0f / (1 << j)));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int acc[4];
                mma_s8u8(acc, ap[0], bv[0][0][h] & (0x01010101u << j), bv[0][1][h] & (0x01010101u << j), start);
#pragma unroll
                for (int z = 1; z < PK; ++z) mma_s8u8(acc, ap[z], bv[z][0][h] & (0x01010101u << j), bv[z][1][h] & (0x01010101u << j));
                o[8 * h + j] = fma2(fma2(pack2(65536.0f, 65536.0f), sums2(acc[0], acc[1]), sums2(acc[2], acc[3])), f, fma2(o[8 * h + j], corr_2, base_2));
            }
        }
    }

    // this warp's tokens together: sums over the lanes of a row, then over the warps through shared memory (the stages' memory, once the copies are done)
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float (*s_o)[ROWS][AMQ_MAX_HEAD_DIM] = reinterpret_cast<float (*)[ROWS][AMQ_MAX_HEAD_DIM]>(smem_raw);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float v0, v1;
        unpack2(o[j], v0, v1);
        v0 += __shfl_xor_sync(0xffffffffu, v0, 16);
        v1 += __shfl_xor_sync(0xffffffffu, v1, 16);
        if (upper) { s_o[warp][r][32 * c + j] = v0; s_o[warp][r][32 * c + 16 + j] = v1; }
    }
    if (lane < 16 && c == 0) { s_m[warp][r] = m; s_l[warp][r] = l; }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        const int rho = rb * ROWS + q;
        if (rho >= p.rows) break;
        const float M = fmaxf(fmaxf(s_m[0][q], s_m[1][q]), fmaxf(s_m[2][q], s_m[3][q])), m_ref = M == -INFINITY ? 0.0f : M;
        float total = 0.0f, v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = exp2_approx(s_m[w][q] - m_ref);
            total += s_l[w][q] * f;
            v += s_o[w][q][threadIdx.x] * f;
        }
        const size_t orow = ((size_t)b * p.q_len + rho / p.group) * p.q_heads + kv * p.group + rho % p.group;
        if (p.splits == 1) {
            if ((int)threadIdx.x < cv.d) p.out[orow * cv.d + threadIdx.x] = total == 0.0f ? 0.0f : v / total;
        } else {
            p.part[(orow * p.splits + split) * AMQ_MAX_HEAD_DIM + threadIdx.x] = v;
            if (threadIdx.x == 0) p.part_ml[orow * p.splits + split] = make_float2(M, total);
        }
    }
}

// joins the shares of a query row: one CTA per row
__global__ void __launch_bounds__(AMQ_MAX_HEAD_DIM)
cache_attention_join_kernel(const float* part, const float2* part_ml, int splits, int d, float* out)
{
    grid_dependency_wait();
    const size_t row = blockIdx.x;
    float M = -INFINITY;
    for (int s = 0; s < splits; ++s) M = fmaxf(M, __ldcg(part_ml + row * splits + s).x);
    const float m_ref = M == -INFINITY ? 0.0f : M;
    float total = 0.0f, v = 0.0f;
    for (int s = 0; s < splits; ++s) {
        const float2 ml = __ldcg(part_ml + row * splits + s);
        const float f = exp2_approx(ml.x - m_ref);
        total += ml.y * f;
        v += __ldcg(part + (row * splits + s) * AMQ_MAX_HEAD_DIM + threadIdx.x) * f;
    }
    if ((int)threadIdx.x < d) out[row * d + threadIdx.x] = total == 0.0f ? 0.0f : v / total;
}

struct AttentionPlan { int rows, row_blocks, splits; size_t part_bytes, bytes; };

AttentionPlan attention_plan(int batch, int q_len, int q_heads, int heads, long long max_tokens)
{
    AttentionPlan a{};
    a.rows = q_len * (q_heads / heads);
    a.row_blocks = (a.rows + ROWS - 1) / ROWS;
    const long long base = (long long)batch * heads * a.row_blocks;
    long long splits = (1184 + base - 1) / base;
    const long long most = (max_tokens + 511) / 512;
    if (splits > most) splits = most;
    if (splits > 128) splits = 128;
    a.splits = splits < 1 ? 1 : (int)splits;
    if (a.splits > 1) {
        const size_t n = (size_t)batch * q_len * q_heads * a.splits;
        a.part_bytes = n * AMQ_MAX_HEAD_DIM * 4;
        a.bytes = a.part_bytes + n * sizeof(float2);
    }
    return a;
}

template <int K>
amq_status launch_attention(const AttentionParams& p, unsigned grid, cudaStream_t st)
{
    constexpr size_t smem = WARPS * (sizeof(Stage<K>) * STAGES + sizeof(Coefficients<K>));
    static_assert(smem >= sizeof(float) * WARPS * ROWS * AMQ_MAX_HEAD_DIM, "the partial sums take the stages' place");
    AMQ_CUDA_TRY(cudaFuncSetAttribute(cache_attention_kernel<K>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    AMQ_CUDA_TRY(launch_kernel(cache_attention_kernel<K>, dim3(grid), dim3(WARPS * 32), smem, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

amq_status cache_view(const uint32_t* kcodes, const float* kcoeffs, const uint32_t* vcodes, const float* vcoeffs, int pages, int page_size, int heads,
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
    if (batch < 1 || q_len < 1 || q_heads < 1 || heads < 1 || q_heads % heads || d < 1 || d > AMQ_MAX_HEAD_DIM || max_tokens < 1) return 0;
    return amq::attention_plan(batch, q_len, q_heads, heads, max_tokens).bytes;
}

amq_status amq_cache_attention(const float* q, long long q_batch, long long q_token, long long q_head,
                               const uint32_t* cache_kcodes, const float* cache_kcoeffs, const uint32_t* cache_vcodes, const float* cache_vcoeffs,
                               int pages, int page_size, int heads, int d, int k, const int32_t* table, int ld_table, int max_pages,
                               const int32_t* lengths, int batch, int q_len, int q_heads, float scale, float* out,
                               void* workspace, size_t workspace_bytes, void* stream)
{
    amq::AttentionParams p{};
    amq_status s = amq::cache_view(cache_kcodes, cache_kcoeffs, cache_vcodes, cache_vcoeffs, pages, page_size, heads, d, k, table, ld_table, max_pages,
                                   lengths, &p.c);
    if (s != AMQ_OK) return s;
    if (batch < 0 || q_len < 0 || q_heads < 1 || q_heads % heads) return AMQ_ERR_INVALID_ARG;
    if ((long long)batch * q_len * q_heads > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (batch == 0 || q_len == 0) return AMQ_OK;
    if (!q || !out || !lengths || (max_pages > 0 && !table)) return AMQ_ERR_INVALID_ARG;
    if (pages > 0 && (!cache_kcodes || !cache_kcoeffs || !cache_vcodes || !cache_vcoeffs)) return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(cache_kcodes) || !amq::aligned16(cache_vcodes)) return AMQ_ERR_ALIGNMENT;
    const amq::AttentionPlan plan = amq::attention_plan(batch, q_len, q_heads, heads, (long long)max_pages * page_size);
    const long long grid = (long long)batch * heads * plan.row_blocks * plan.splits;
    if (grid > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (plan.bytes) {
        if (!workspace || workspace_bytes < plan.bytes) return AMQ_ERR_WORKSPACE;
        if (!amq::aligned16(workspace)) return AMQ_ERR_ALIGNMENT;
    }
    p.q = q; p.q_batch = q_batch; p.q_token = q_token; p.q_head = q_head;
    p.q_len = q_len; p.q_heads = q_heads; p.group = q_heads / heads; p.scale = scale; p.out = out;
    p.rows = plan.rows; p.row_blocks = plan.row_blocks; p.splits = plan.splits;
    p.part = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + plan.part_bytes);
    p.wide = amq::aligned16(cache_kcoeffs) && amq::aligned16(cache_vcoeffs);
    cudaStream_t st = (cudaStream_t)stream;
    switch (k) {
        case 1: s = amq::launch_attention<1>(p, (unsigned)grid, st); break;
        case 2: s = amq::launch_attention<2>(p, (unsigned)grid, st); break;
        case 3: s = amq::launch_attention<3>(p, (unsigned)grid, st); break;
        default: s = amq::launch_attention<4>(p, (unsigned)grid, st); break;
    }
    if (s != AMQ_OK || plan.splits == 1) return s;
    AMQ_CUDA_TRY(amq::launch_kernel(amq::cache_attention_join_kernel, dim3((unsigned)(batch * q_len * q_heads)), dim3(AMQ_MAX_HEAD_DIM), 0, st, true, p.part, p.part_ml,
                                    plan.splits, d, out));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // extern "C"
