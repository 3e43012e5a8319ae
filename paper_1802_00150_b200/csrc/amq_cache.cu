// A paged cache that holds keys and values in packed planes, as the row quantizer leaves them: writing of new rows, and attention over it.
//
//   s[t] = scale * sum_i a[t][i] (q . b[t][i]),   p = softmax over the visible t,   o = sum_t p[t] sum_i a'[t][i] b'[t][i]
// with the planes b, b' (+-1) and coefficients a, a' of token t's key and value.
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

template <int BYTES> __device__ __forceinline__ void copy_async(void* to, const void* from, bool real)
{
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
    const int n = real ? BYTES : 0;                 // (nothing is read for the others: zeros are written)
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(from), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" :: "r"(dst), "l"(from), "r"(n), "n"(BYTES) : "memory");
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

__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

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
    const CacheView& cv = p.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3, r = g & 3;
    const bool upper = g < 4;           // rows g, g + 8: digits 3 and 1 of the query (weights: 2 and 0), else 2 and 0 (1 and none)
    Stage<K>* stages = reinterpret_cast<Stage<K>*>(smem_raw) + warp * STAGES;
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
    const size_t step = (size_t)cv.heads * K;
    const uint4* const kcodes = reinterpret_cast<const uint4*>(cv.kcodes) + (size_t)kv * K;
    const uint4* const vcodes = reinterpret_cast<const uint4*>(cv.vcodes) + (size_t)kv * K;
    const float *const kcoeffs = cv.kcoeffs + (size_t)kv * K, *const vcoeffs = cv.vcoeffs + (size_t)kv * K;
    auto issue = [&](Stage<K>& st, int slot) {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int idx = i * 32 + lane, token = idx / K, plane = idx % K;
            const int s = __shfl_sync(0xffffffffu, slot, token);
            const size_t from = (size_t)max(s, 0) * step + plane;
            copy_async<16>(&st.k[place<K>(token, plane)], kcodes + from, s >= 0);
            copy_async<16>(&st.v[place<K>(token, plane)], vcodes + from, s >= 0);
        }
        const size_t from = (size_t)max(slot, 0) * step;
        float *ka = st.ka + lane * pitch(K), *va = st.va + lane * pitch(K);
        constexpr int UNIT = K == 3 ? 1 : K;
        if (p.wide) {
#pragma unroll
            for (int i = 0; i < K; i += UNIT) {
                copy_async<4 * UNIT>(ka + i, kcoeffs + from + i, slot >= 0);
                copy_async<4 * UNIT>(va + i, vcoeffs + from + i, slot >= 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i) {
                copy_async<4>(ka + i, kcoeffs + from + i, slot >= 0);
                copy_async<4>(va + i, vcoeffs + from + i, slot >= 0);
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
        if (real[s]) issue(stages[s], now);
        commit();
    }

    // the query's digits as the MMAs take them, and the digits' sums (times the bytes' weights) over the row
    uint32_t aq[4][4];
    float half_sum[2], factor;
    {
        float x[32];
        uint32_t largest = 0;
        const int i = row / p.group, h = kv * p.group + row % p.group;
        const float* q = p.q + b * p.q_batch + i * p.q_token + h * p.q_head + 32 * c;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            x[j] = row < p.rows && 32 * c + j < cv.d ? q[j] : 0.0f;
            largest = max(largest, __float_as_uint(x[j]) & 0x7fffffffu);
        }
        largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
        largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
        const int e = max((int)(largest >> 23), 29);
        const bool finite = largest < 0x7f800000u;
        const float to_fixed = finite ? __int_as_float((283 - e) << 23) : 0.0f;         // largest element below 2^30
        int sum[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t a0 = 0, a1 = 0;
#pragma unroll
            for (int byte = 0; byte < 4; ++byte) {
                const uint32_t y = (uint32_t)__float2int_rn(x[j + 8 * byte] * to_fixed * (1.0f / (1 << j))) + 0x80808080u;
                const int d0 = (int)((upper ? y >> 24 : y >> 16) & 255u) - 128, d1 = (int)((upper ? y >> 8 : y) & 255u) - 128;
                a0 |= (uint32_t)(d0 & 255) << (8 * byte);
                a1 |= (uint32_t)(d1 & 255) << (8 * byte);
                sum[0] += d0 * (1 << j); sum[1] += d1 * (1 << j);
            }
            aq[j >> 1][(j & 1) * 2] = a0;
            aq[j >> 1][(j & 1) * 2 + 1] = a1;
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 1);
            sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 2);
            half_sum[w] = 0.5f * (float)sum[w];
        }
        factor = finite ? 1.0f / to_fixed * p.scale * (2.0f * 1.44269504f) : NAN;       // scores in units of log 2
    }
    const float w0 = upper ? 16777216.0f : 65536.0f, w1 = upper ? 256.0f : 1.0f;        // digits' weights: keys
    const float wv = upper ? 65536.0f : 256.0f;                                         // values (row g + 8: 1 or nothing)
    const f32x2 w0_2 = pack2(w0, w0), w1_2 = pack2(w1, w1), wv_2 = pack2(wv, wv);
    const f32x2 minus_half0 = pack2(-half_sum[0], -half_sum[0]), minus_half1 = pack2(-half_sum[1], -half_sum[1]);
    const uint32_t sel = upper ? 0x62u : 0x51u, keep = upper ? 0xffffffffu : 0u;
    const uint32_t half = g & 1 ? 0x7362u : 0x5140u;        // bytes of the plane words that hold dimensions 16 g ..
    int start[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("mov.b32 %0, 0x4B400000;" : "=r"(start[i]));

    float m = -INFINITY, l = 0.0f;
    f32x2 o[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) o[j] = pack2(0.0f, 0.0f);

    int stage = 0;
    for (; tile < tile1; tile += WARPS) {
        {
            const int now = slot;
            slot = slot_at(tile + STAGES * WARPS);
            real[STAGES - 1] = __ballot_sync(0xffffffffu, now >= 0);
            __syncwarp();
            if (real[STAGES - 1]) issue(stages[stage == 0 ? STAGES - 1 : stage - 1], now);
            commit();
            asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 1) : "memory");
            __syncwarp();
        }
        const Stage<K>& st = stages[stage];
        const uint32_t on_a_page = real[0];
#pragma unroll
        for (int q = 0; q < STAGES - 1; ++q) real[q] = real[q + 1];
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (on_a_page == 0) continue;           // (nothing was copied)
        // tokens that this lane's row sees
        const int left = my_limit - tile * TILE;
        const uint32_t seen = on_a_page & (left >= TILE ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u);

        // The coefficients by planes, so that those of tokens 2 c, 2 c + 1 lie together; the values' largest decides the fixed point of the tile's
        // weights.  (What lanes read of the last tile they have read: the shuffles of its maximum lie behind.)
        uint32_t largest = 0;
        float va[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            coef.k[i][lane] = st.ka[lane * pitch(K) + i];
            va[i] = st.va[lane * pitch(K) + i];
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
        const int ev = max((int)(largest >> 23), 22);
        const float to_fixed = __int_as_float((275 - ev) << 23), from_fixed = __int_as_float((ev - 21) << 23);

        // scores of tokens 8 n + 2 c, 8 n + 2 c + 1
        float s[4][2];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            f32x2 x = 0, y = 0, all = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                int acc[4];
                const uint32_t w = reinterpret_cast<const uint32_t*>(&st.k[place<K>(8 * n + g, i)])[c];
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
                if (i >= K) { y[2 * n][i] = y[2 * n + 1][i] = 0x00808080u; word[2 * n][i] = word[2 * n + 1][i] = 0u; continue; }
                const int j = i < K ? i : 0;
                float f0, f1;
                unpack2(fma2(ws, *reinterpret_cast<const f32x2*>(&coef.v[j][8 * n + 2 * c]), pack2(MAGIC, MAGIC)), f0, f1);
                y[2 * n][i] = (uint32_t)__float_as_int(f0) + (0x00808080u - (uint32_t)MAGIC_BITS);
                y[2 * n + 1][i] = (uint32_t)__float_as_int(f1) + (0x00808080u - (uint32_t)MAGIC_BITS);
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    word[2 * n + e][i] = reinterpret_cast<const uint32_t*>(&st.v[place<K>(8 * n + 2 * c + e, j)])[g >> 1];
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
                ap[z][2 * side] = __byte_perm(__byte_perm(yy[0], yy[1], sel), __byte_perm(yy[2], yy[3], sel), 0x5410) ^ 0x80808080u;
                ap[z][2 * side + 1] = (__byte_perm(__byte_perm(yy[0], yy[1], 0x40), __byte_perm(yy[2], yy[3], 0x40), 0x5410) ^ 0x80808080u) & keep;
                const uint32_t t0 = __byte_perm(ww[0], ww[1], half), t1 = __byte_perm(ww[2], ww[3], half);
                bv[z][side][0] = __byte_perm(t0, t1, 0x5410);
                bv[z][side][1] = __byte_perm(t0, t1, 0x7632);
            }
        l = fmaf(l, corr, sum * tile_factor);
        int ones[4];
        mma_s8u8(ones, ap[0], 0x01010101u, 0x01010101u, start);
#pragma unroll
        for (int z = 1; z < PK; ++z) mma_s8u8(ones, ap[z], 0x01010101u, 0x01010101u);
        const float unit = tile_factor * from_fixed;
        const float base = -unit * fmaf(wv, __int_as_float(ones[0]) - MAGIC, __int_as_float(ones[2]) - MAGIC);
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
                o[8 * h + j] = fma2(fma2(wv_2, sums2(acc[0], acc[1]), sums2(acc[2], acc[3])), f, fma2(o[8 * h + j], corr_2, base_2));
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
