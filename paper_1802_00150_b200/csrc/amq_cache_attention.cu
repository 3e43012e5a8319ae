// Attention over a paged cache in packed planes (amq_cache.cuh):
//
//   s[t] = scale * sum_i a[t][i] (q . b[t][i]),   p = softmax over the visible t,   o = sum_t p[t] sum_i a'[t][i] b'[t][i]
//
// with the planes b, b' (+-1) and coefficients a, a' of token t's key and value.
#include <stddef.h>

#include "amq_cache.cuh"
#include "amq_pairs.cuh"

namespace amq {
namespace {

struct AttentionParams {
    CacheView c;
    const float* q; long long q_batch, q_token, q_head;
    int q_len, q_heads, group;
    int rows, row_blocks;               // query rows of a key head: q_len * group, in blocks
    int batch;
    int shares;                         // 0: a CTA takes a block's whole sequence; else the tiles of all are dealt out to so many CTAs for each block
    bool wide;                          // coefficient rows on their own size (4, 8 or 16 bytes)
    float scale;
    float* out;
    float* part; float2* part_ml;       // of the blocks that a share's edge cuts: unnormalised results and {maximum, sum}, [CTA][2][row of the block]
};

constexpr int TILE = 32;                // tokens
constexpr int STAGES = 2;
constexpr int ROWS = 4;                 // query rows of a row tile
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

// Loads under a predicate, -1 or 0 where it does not hold.  (As a conditional expression the compiler moves the loaded value behind a branch, and
// waits for it there.)
__device__ __forceinline__ int load_page(const int32_t* from, bool real)
{
    int v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.b32 %0, -1;\n\t@p ld.global.b32 %0, [%1];\n\t}"
                 : "=&r"(v) : "l"(from), "r"((uint32_t)real) : "memory");
    return v;
}

__device__ __forceinline__ float load_float(const float* from, bool real)
{
    float v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\tmov.f32 %0, 0f00000000;\n\t@p ld.global.f32 %0, [%1];\n\t}"
                 : "=&f"(v) : "l"(from), "r"((uint32_t)real) : "memory");
    return v;
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

// One instruction, within 2^-22 of itself, as exp2f is not: a weight's error then is that of its score (whose fp32 sum of some hundred terms is off by as much
// and more), and exp2f would add instructions to a kernel that is bound by them.
__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

__device__ __forceinline__ int tiles_of(const CacheView& c, int b) { const int n = visible_length(c, b); return n > 0 ? (n - 1) / TILE + 1 : 0; }

// The tiles of all sequences in a line, one behind the other: share s of n has those from total s / n on, so that CTAs have the same work whatever the lengths.
// Each of the `units` blocks of a sequence (key heads and their row blocks) has its own n shares, and CTAs that follow one another are at the same tokens of
// different heads, whose rows lie side by side in the cache.  Found by each warp on its own.
__device__ __forceinline__ long long total_tiles(const AttentionParams& p)
{
    const int lane = threadIdx.x & 31;
    int n = 0;
    long long total = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        n = b0 + lane < p.batch ? tiles_of(p.c, b0 + lane) : 0;
        total += (long long)__reduce_add_sync(0xffffffffu, (uint32_t)n & 0xffffu) + ((long long)__reduce_add_sync(0xffffffffu, (uint32_t)n >> 16) << 16);
    }
    return total;
}
// The shares that a line of so many tiles goes to: the lengths may be far below what the table has room for, and a share without tiles would leave nothing for the
// second kernel to join.
__device__ __forceinline__ int shares_of(const AttentionParams& p, long long total) { return (int)min((long long)p.shares, (total + 3) / 4); }

// the sequence that holds place x of the line (x below the total), and the tiles in front of it
__device__ __forceinline__ int sequence_at(const AttentionParams& p, long long x, long long* before)
{
    const int lane = threadIdx.x & 31;
    long long front = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
        const long long n = b0 + lane < p.batch ? tiles_of(p.c, b0 + lane) : 0;
        long long sum = n;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long o = __shfl_up_sync(0xffffffffu, sum, off);
            if (lane >= off) sum += o;
        }
        const long long at = front + sum - n;
        const uint32_t here = __ballot_sync(0xffffffffu, at <= x && x < at + n);
        if (here) {
            const int l = __ffs(here) - 1;
            *before = __shfl_sync(0xffffffffu, at, l);
            return b0 + l;
        }
        front += __shfl_sync(0xffffffffu, sum, 31);
    }
    *before = front;
    return p.batch;
}

// The products run on the integer tensor cores, on the planes' bits as they are stored: a word ANDed with 0x01010101 << j is four bytes of 0 or
// 2^j, an operand of mma.m16n8k32 with the query (or the weights) as digits of eight bits.  A query row is four rows of the operand, its
// digits, so that four query rows fill the 16 rows of an instruction, and the product is exact:
//   q = sum_digits 256^i d_i (31-bit fixed point; elements whose bits lie at position j of a byte are held divided by 2^j),
//   q . b = 2 sum_{bit = 1} q - sum q.
// What bounds the kernel is the issue of instructions: for 8 tokens of 4 bits 33 MMAs, each of which takes 2.2 clocks of an SM, 8.8 of a scheduler, and hides
// half at most of what stands beside it (3.3 with two logic and four fp32 instructions, which alone take 2.0), and 300 others (64 AND, 36 byte permutations, 60 two-wide fp32, 36 of shared memory, 12 of
// exponentials and conversions), against 1280 bytes.  64 sequences of 1024 to 4096 tokens, 8 heads, 32 query heads, d = 128, 4 bits: 111 us, 1.9 TB/s
// (plain kernel, a CTA to a query row: 3346 us).  With the products on tcgen05 (kind::i8: keys' bytes in tensor memory, values' in shared memory, dimensions
// contiguous) the same took 167 us: 7060 instructions for 128 tokens, nearly as many, and a chain of 5800 clocks from scores to results.
//
// A warp takes tiles of 32 tokens on its own (its copies, through a ring of its own stages; the softmax's running maximum and sum; partial sums), the
// CTA's warps are joined at the end, and the pieces of a block that a share's edge cuts by a second kernel.
//
// Lane l = 4 g + c of an MMA holds rows g and g + 8: digits g / 4 and 2 + g / 4 of query row g mod 4.  For keys, column g is token g of eight and c the
// word of the plane; results are those of tokens 2 c, 2 c + 1.  For values, c stands for the same two tokens, so weights never change
// lanes, and column g for dimensions 16 g .. 16 g + 15, one per MMA.
//
// MT: row tiles of a CTA; what is done with the planes is done once for all of them.  WARPS: of a CTA.  (Four warps, one row tile: 128 registers for four CTAs an SM;
// at 4 bits 88 bytes of them are spilled, at 2 and 3 some 25.)
template <int K, int MT, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, WARPS > 4 ? 1 : MT == 1 ? 4 : 2)
cache_attention_kernel(const __grid_constant__ AttentionParams p)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    constexpr int BLOCK = ROWS * MT;
    __shared__ float s_m[WARPS][BLOCK], s_l[WARPS][BLOCK];
    __shared__ uint32_t s_largest[4][BLOCK];
    __shared__ uint4 s_digits[4][MT][32];
    __shared__ int s_sum[4][MT][8][2];
    const CacheView& cv = p.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3, r = g & 3;
    const bool upper = g < 4;           // rows g, g + 8: digits 3 and 1, else 2 and 0
    const uint32_t digit0 = upper ? 0x73u : 0x62u, digit1 = upper ? 0x51u : 0x40u;      // these bytes of two words
    Stage<K>* stages = reinterpret_cast<Stage<K>*>(smem_raw) + warp * STAGES;
    const uint32_t stage_at = (uint32_t)__cvta_generic_to_shared(stages);
    Coefficients<K>& coef = (reinterpret_cast<Coefficients<K>*>(reinterpret_cast<Stage<K>*>(smem_raw) + WARPS * STAGES))[warp];

    const uint32_t step = (uint32_t)cv.heads * K;           // planes of a token (at most 2^18)
    const int units = cv.heads * p.row_blocks;

    grid_dependency_wait();
    // this CTA's pieces: one block's whole sequence, or those of its share of the line
    const int block = blockIdx.x % units, rb = block % p.row_blocks, kv = block / p.row_blocks, share = blockIdx.x / units;
    int b = share, tiles;
    long long x = 0, x1 = 1, before = 0;
    if (p.shares) {
        const long long total = total_tiles(p);
        const int shares = shares_of(p, total);
        if (share >= shares) return;
        x = total * share / shares;
        x1 = total * (share + 1) / shares;
        b = sequence_at(p, x, &before);
    }
    tiles = tiles_of(cv, b);
  for (;;) {
    int tile0 = 0, tile1 = tiles;
    if (p.shares) {
        tile0 = (int)(x - before);
        tile1 = (int)min((long long)tiles, tile0 + (x1 - x));
    }
    const int length = visible_length(cv, b);
    const int last_row = min(rb * BLOCK + BLOCK, p.rows) - 1;
    const int limit = max(length - p.q_len + 1 + last_row / p.group, 0);        // of the block's last row: no other sees more
    int my_limit[MT];                   // tokens that this lane's rows see
#pragma unroll
    for (int z = 0; z < MT; ++z) {
        const int row = rb * BLOCK + z * ROWS + r;
        my_limit[z] = row < p.rows ? length - p.q_len + 1 + row / p.group : limit;
    }
    // the query's elements that this warp turns into digits, on their way with the first tiles
    float xq[MT][8];
    if (warp < 4) {
#pragma unroll
        for (int z = 0; z < MT; ++z) {
            const int row = rb * BLOCK + z * ROWS + r, i = row / p.group, h = kv * p.group + row % p.group, first = 32 * c + 2 * warp;
            const float* q = p.q + b * p.q_batch + i * p.q_token + h * p.q_head + first;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int dim = 8 * (e >> 1) + (e & 1);
                xq[z][e] = load_float(q + dim, row < p.rows && first + dim < cv.d);
            }
        }
    }

    // a tile's pages, a token a lane, as the table has them (-1 behind the last token), and the slots from that: two steps, a tile apart
    auto page_at = [&](int tile) {
        const int t = tile * TILE + lane;
        const bool real = tile < tile1 && t < limit;
        return load_page(cv.table + (size_t)b * cv.ld_table + (real ? page_index(cv, t) : 0), real);
    };
    // planes: K lanes a token, so that an instruction's lanes meet few lines; coefficients: a lane a token
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
    int page = page_at(tile);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        const int now = slot_on(cv, page, (tile + s * WARPS) * TILE + lane);
        page = page_at(tile + (s + 1) * WARPS);
        real[s] = __ballot_sync(0xffffffffu, now >= 0);
        if (real[s]) issue(stage_at + s * (uint32_t)sizeof(Stage<K>), now);
        commit();
    }

    // The query's digits as the MMAs take them, and the digits' sums (times the bytes' weights) over the row.  A warp makes those of two bit positions.
    uint32_t aq[MT][4][4];
    float half_sum[MT][2], factor[MT];
    {
        if (warp < 4) {
#pragma unroll
            for (int z = 0; z < MT; ++z) {
                uint32_t largest = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) largest = max(largest, __float_as_uint(xq[z][e]) & 0x7fffffffu);
                largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 1));
                largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, 2));
                if (upper && c == 0) s_largest[warp][z * ROWS + r] = largest;
            }
        }
        __syncthreads();
#pragma unroll
        for (int z = 0; z < MT; ++z) {
            const int at_row = z * ROWS + r;
            const uint32_t largest = max(max(s_largest[0][at_row], s_largest[1][at_row]), max(s_largest[2][at_row], s_largest[3][at_row]));
            const int e = max((int)(largest >> 23), 29);
            const bool finite = largest < 0x7f800000u;
            const float to_fixed = finite ? __int_as_float((283 - e) << 23) : 0.0f;         // largest element below 2^30
            factor[z] = finite ? 1.0f / to_fixed * p.scale * (2.0f * 1.44269504f) : NAN;    // scores in units of log 2
            if (warp < 4) {
                const float to_fixed_here = to_fixed * __int_as_float((127 - 2 * warp) << 23);
                int sum[2] = {0, 0};
                uint32_t a[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t y[4];
#pragma unroll
                    for (int byte = 0; byte < 4; ++byte) {
                        y[byte] = (uint32_t)__float2int_rn(xq[z][2 * byte + j] * to_fixed_here * (j ? 0.5f : 1.0f)) + 0x80808080u;
#pragma unroll
                        for (int w = 0; w < 2; ++w) sum[w] += ((int)(__byte_perm(y[byte], 0, w ? digit1 & 0x7u : digit0 & 0x7u) & 255u) - 128) * (1 << j);
                    }
                    a[2 * j] = __byte_perm(__byte_perm(y[0], y[1], digit0), __byte_perm(y[2], y[3], digit0), 0x5410) ^ 0x80808080u;
                    a[2 * j + 1] = __byte_perm(__byte_perm(y[0], y[1], digit1), __byte_perm(y[2], y[3], digit1), 0x5410) ^ 0x80808080u;
                }
                s_digits[warp][z][lane] = make_uint4(a[0], a[1], a[2], a[3]);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 1);
                    sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], 2);
                    if (c == 0) s_sum[warp][z][g][w] = sum[w] * (1 << (2 * warp));
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int z = 0; z < MT; ++z) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 d = s_digits[j][z][lane];
                aq[z][j][0] = d.x; aq[z][j][1] = d.y; aq[z][j][2] = d.z; aq[z][j][3] = d.w;
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) half_sum[z][w] = 0.5f * (float)(s_sum[0][z][g][w] + s_sum[1][z][g][w] + s_sum[2][z][g][w] + s_sum[3][z][g][w]);
        }
    }
    const float w0 = upper ? 16777216.0f : 65536.0f, w1 = upper ? 256.0f : 1.0f;        // the digits' weights
    const f32x2 w0_2 = pack2(w0, w0), w1_2 = pack2(w1, w1);
    const uint32_t half = g & 1 ? 0x7362u : 0x5140u;        // bytes of the plane words that hold dimensions 16 g ..
    int start[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("mov.b32 %0, %1;" : "=r"(start[i]) : "n"(MAGIC_BITS));

    float m[MT], l[MT];
    f32x2 o[MT][16];
#pragma unroll
    for (int z = 0; z < MT; ++z) {
        m[z] = -INFINITY; l[z] = 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) o[z][j] = pack2(0.0f, 0.0f);
    }

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
            const int now = slot_on(cv, page, (tile + (STAGES - 1) * WARPS) * TILE + lane);
            page = page_at(tile + STAGES * WARPS);
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
        // tokens that this lane's rows see
        uint32_t seen[MT];
#pragma unroll
        for (int z = 0; z < MT; ++z) {
            const int left = my_limit[z] - tile * TILE;
            seen[z] = on_a_page & (left >= TILE ? 0xffffffffu : left > 0 ? (1u << left) - 1u : 0u);
        }

        // The coefficients by planes, so that those of tokens 2 c, 2 c + 1 lie together; the values' largest decides the fixed point of the tile's
        // weights.  (The barrier behind the copies lies behind everybody's reading of the last tile's.)
        uint32_t mine = 0, mine_k = 0;          // of this lane's token
        float va[K];
        float ka[K];
        load_row<K>(st.ka + lane * pitch(K), ka);
        load_row<K>(st.va + lane * pitch(K), va);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            coef.k[i][lane] = ka[i];
            mine = max(mine, __float_as_uint(va[i]) & 0x7fffffffu);
            mine_k = max(mine_k, __float_as_uint(ka[i]) & 0x7fffffffu);
        }
        uint32_t largest = __reduce_max_sync(0xffffffffu, mine_k >= 0x7f800000u ? mine_k : mine);
        if (largest >= 0x7f800000u) {           // NaN or infinite coefficients: they count for the rows that see them, and for those only
            bool bad = mine_k >= 0x7f800000u;
            mine = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                if (!isfinite(va[i])) { bad = true; va[i] = 0.0f; }
                mine = max(mine, __float_as_uint(va[i]) & 0x7fffffffu);
            }
            largest = __reduce_max_sync(0xffffffffu, mine);
            const uint32_t all_bad = __ballot_sync(0xffffffffu, bad);
#pragma unroll
            for (int z = 0; z < MT; ++z)
                if (all_bad & seen[z]) l[z] = NAN;
        }
#pragma unroll
        for (int i = 0; i < K; ++i) coef.v[i][lane] = va[i];
        // Where rows of the block see different tokens (the last tiles of a call with several queries a sequence), each goes by the largest of those that it
        // sees: a later query's token would take bits from the earlier ones' weights.
        uint32_t size[MT];
        bool differ = false;
#pragma unroll
        for (int z = 0; z < MT; ++z) { size[z] = largest; differ |= seen[z] != on_a_page; }
        if (__any_sync(0xffffffffu, differ)) {
#pragma unroll
            for (int z = 0; z < MT; ++z)
#pragma unroll
                for (int row = 0; row < ROWS; ++row) {
                    const uint32_t tokens = __shfl_sync(0xffffffffu, seen[z], 4 * row), of_row = __reduce_max_sync(0xffffffffu, tokens >> lane & 1 ? mine : 0u);
                    if (r == row) size[z] = of_row;
                }
        }
        __syncwarp();
        float to_fixed[MT];                     // products below 2^30
#pragma unroll
        for (int z = 0; z < MT; ++z) to_fixed[z] = __int_as_float((283 - max((int)(size[z] >> 23), 30)) << 23);

        // scores of tokens 8 n + 2 c, 8 n + 2 c + 1
        float s[MT][4][2];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            // (chains of four MMAs, those of the planes side by side)
            uint32_t word[K];
            int acc[K][MT][4];
#pragma unroll
            for (int i = 0; i < K; ++i) word[i] = *reinterpret_cast<const uint32_t*>(words + kat[i] + n * 8 * pitch(K) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    const uint32_t b0 = word[i] & (0x01010101u << (2 * j)), b1 = word[i] & (0x02020202u << (2 * j));
#pragma unroll
                    for (int z = 0; z < MT; ++z) {
                        if (j == 0) mma_s8u8(acc[i][z], aq[z][j], b0, b1, start);
                        else mma_s8u8(acc[i][z], aq[z][j], b0, b1);
                    }
                }
            f32x2 x[MT], y[MT], all = 0;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const f32x2 a = *reinterpret_cast<const f32x2*>(&coef.k[i][8 * n + 2 * c]);
#pragma unroll
                for (int z = 0; z < MT; ++z) {
                    x[z] = i ? fma2(a, sums2(acc[i][z][0], acc[i][z][1]), x[z]) : mul2(a, sums2(acc[i][z][0], acc[i][z][1]));
                    y[z] = i ? fma2(a, sums2(acc[i][z][2], acc[i][z][3]), y[z]) : mul2(a, sums2(acc[i][z][2], acc[i][z][3]));
                }
                all = i ? add2(all, a) : a;
            }
#pragma unroll
            for (int z = 0; z < MT; ++z) {
                x[z] = fma2(pack2(-half_sum[z][0], -half_sum[z][0]), all, x[z]);
                y[z] = fma2(pack2(-half_sum[z][1], -half_sum[z][1]), all, y[z]);
                unpack2(fma2(w0_2, x[z], mul2(w1_2, y[z])), s[z][n][0], s[z][n][1]);
#pragma unroll
                for (int e = 0; e < 2; ++e) s[z][n][e] = (s[z][n][e] + __shfl_xor_sync(0xffffffffu, s[z][n][e], 16)) * factor[z];
            }
        }
        // the values' planes: K MMA steps, in whose 32 positions this lane's are the planes of its eight tokens, eight planes a step
        uint32_t bv[K][2][2];
        {
            uint32_t word[8 * K];               // by this lane's tokens, (n, e) = (0, 0), (0, 1), (1, 0), .., and planes
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int i = 0; i < K; ++i) word[q * K + i] = *reinterpret_cast<const uint32_t*>(words + vat[i] + ((q >> 1) * 8 + (q & 1)) * pitch(K) * 16);
#pragma unroll
            for (int z = 0; z < K; ++z)
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const uint32_t* const ww = word + (2 * z + side) * 4;
                    const uint32_t t0 = __byte_perm(ww[0], ww[1], half), t1 = __byte_perm(ww[2], ww[3], half);
                    bv[z][side][0] = __byte_perm(t0, t1, 0x5410);
                    bv[z][side][1] = __byte_perm(t0, t1, 0x7632);
                }
        }
        // weights, relative to the tile's maximum, times coefficients as digits
        uint32_t ap[MT][K][4];
        float unit[MT];
        f32x2 base_2[MT], corr_2[MT];
#pragma unroll
        for (int z = 0; z < MT; ++z) {
            if (__any_sync(0xffffffffu, seen[z] != 0xffffffffu)) {
                const uint32_t mine = seen[z] >> (2 * c);
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) s[z][n][e] = mine >> (8 * n + e) & 1 ? s[z][n][e] : -INFINITY;
            }
            float top = s[z][0][0];
#pragma unroll
            for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(s[z][n][0], s[z][n][1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float ref = top == -INFINITY ? 0.0f : top, m_new = fmaxf(m[z], top), m_ref = m_new == -INFINITY ? 0.0f : m_new;
            const float corr = exp2_approx(m[z] - m_ref), tile_factor = exp2_approx(top - m_ref);
            m[z] = m_new;
            float sum = 0.0f;
            uint32_t y[8 * K];                  // by this lane's tokens and planes
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float e0 = exp2_approx(s[z][n][0] - ref), e1 = exp2_approx(s[z][n][1] - ref);
                sum += e0 + e1;
                const f32x2 ws = mul2(pack2(e0, e1), pack2(to_fixed[z], to_fixed[z]));
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    float f0, f1;
                    unpack2(mul2(ws, *reinterpret_cast<const f32x2*>(&coef.v[i][8 * n + 2 * c])), f0, f1);
                    y[2 * n * K + i] = (uint32_t)__float2int_rn(f0) + 0x80808080u;
                    y[(2 * n + 1) * K + i] = (uint32_t)__float2int_rn(f1) + 0x80808080u;
                }
            }
#pragma unroll
            for (int q = 0; q < K; ++q)
#pragma unroll
                for (int side = 0; side < 2; ++side) {
                    const uint32_t* const yy = y + (2 * q + side) * 4;
                    ap[z][q][2 * side] = __byte_perm(__byte_perm(yy[0], yy[1], digit0), __byte_perm(yy[2], yy[3], digit0), 0x5410) ^ 0x80808080u;
                    ap[z][q][2 * side + 1] = __byte_perm(__byte_perm(yy[0], yy[1], digit1), __byte_perm(yy[2], yy[3], digit1), 0x5410) ^ 0x80808080u;
                }
            l[z] = fmaf(l[z], corr, sum * tile_factor);
            int ones[4];
            mma_s8u8(ones, ap[z][0], 0x01010101u, 0x01010101u, start);
#pragma unroll
            for (int q = 1; q < K; ++q) mma_s8u8(ones, ap[z][q], 0x01010101u, 0x01010101u);
            unit[z] = tile_factor * __int_as_float(0x7f000000 - __float_as_int(to_fixed[z])) * w1;         // (1 / to_fixed, a power of two; w0 = 2^16 w1)
            const float base = -unit[z] * fmaf(65536.0f, __int_as_float(ones[0]) - MAGIC, __int_as_float(ones[2]) - MAGIC);
            base_2[z] = pack2(base, base); corr_2[z] = pack2(corr, corr);
        }
        constexpr int SIDE = MT == 1 ? 2 : 1;   // bit positions at once: four chains side by side
#pragma unroll
        for (int j0 = 0; j0 < 8; j0 += SIDE) {
            int acc[SIDE][2][MT][4];
#pragma unroll
            for (int q = 0; q < K; ++q)
#pragma unroll
                for (int s = 0; s < SIDE; ++s)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t b0 = bv[q][0][h] & (0x01010101u << (j0 + s)), b1 = bv[q][1][h] & (0x01010101u << (j0 + s));
#pragma unroll
                        for (int z = 0; z < MT; ++z) {
                            if (q == 0) mma_s8u8(acc[s][h][z], ap[z][q], b0, b1, start);
                            else mma_s8u8(acc[s][h][z], ap[z][q], b0, b1);
                        }
                    }
#pragma unroll
            for (int s = 0; s < SIDE; ++s)
#pragma unroll
                for (int z = 0; z < MT; ++z) {
                    const f32x2 f = pack2(unit[z] * (2.0f / (1 << (j0 + s))), unit[z] * (2.0f / (1 << (j0 + s))));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        f32x2& to = o[z][8 * h + j0 + s];
                        const int (&a)[4] = acc[s][h][z];
                        to = fma2(fma2(pack2(65536.0f, 65536.0f), sums2(a[0], a[1]), sums2(a[2], a[3])), f, fma2(to, corr_2[z], base_2[z]));
                    }
                }
        }
    }

    // this warp's tokens together: sums over the lanes of a row, then, row tile by row tile, over the warps through shared memory (the stages' memory, once
    // the copies are done)
    asm volatile("cp.async.wait_all;" ::: "memory");
    float (*s_o)[ROWS * 4][33] = reinterpret_cast<float (*)[ROWS * 4][33]>(smem_raw);        // (33: the lanes' 32 dimensions on different banks)
#pragma unroll
    for (int z = 0; z < MT; ++z) {
        l[z] += __shfl_xor_sync(0xffffffffu, l[z], 1);
        l[z] += __shfl_xor_sync(0xffffffffu, l[z], 2);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float v0, v1;
            unpack2(o[z][j], v0, v1);
            v0 += __shfl_xor_sync(0xffffffffu, v0, 16);
            v1 += __shfl_xor_sync(0xffffffffu, v1, 16);
            if (upper) { s_o[warp][r * 4 + c][j] = v0; s_o[warp][r * 4 + c][16 + j] = v1; }
        }
        if (lane < 16 && c == 0) { s_m[warp][z * ROWS + r] = m[z]; s_l[warp][z * ROWS + r] = l[z]; }
        __syncthreads();
        for (int at = threadIdx.x; at < ROWS * AMQ_MAX_HEAD_DIM; at += WARPS * 32) {
            const int q = z * ROWS + at / AMQ_MAX_HEAD_DIM, dim = at % AMQ_MAX_HEAD_DIM, rho = rb * BLOCK + q;
            if (rho >= p.rows) break;
            float M = s_m[0][q];
#pragma unroll
            for (int w = 1; w < WARPS; ++w) M = fmaxf(M, s_m[w][q]);
            const float m_ref = M == -INFINITY ? 0.0f : M;
            float total = 0.0f, v = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float f = exp2_approx(s_m[w][q] - m_ref);
                total += s_l[w][q] * f;
                v += s_o[w][at / 32][dim & 31] * f;
            }
            if (tile0 == 0 && tile1 == tiles) {
                const size_t orow = ((size_t)b * p.q_len + rho / p.group) * p.q_heads + kv * p.group + rho % p.group;
                if (dim < cv.d) p.out[orow * cv.d + dim] = total == 0.0f ? 0.0f : v / total;
            } else {                    // (a share has two such pieces at most: one that begins before it, one that ends behind it)
                const size_t part = ((size_t)blockIdx.x * 2 + (tile0 > 0 ? 0 : 1)) * BLOCK + q;
                p.part[part * AMQ_MAX_HEAD_DIM + dim] = v;
                if (dim == 0) p.part_ml[part] = make_float2(M, total);
            }
        }
    }
    if (p.shares == 0) return;
    x += tile1 - tile0;
    if (x >= x1) return;
    before += tiles;                    // (there is more: on to the next sequence that has tiles)
    do tiles = tiles_of(cv, ++b); while (tiles == 0);
    __syncthreads();                    // (the sums have been read, and the digits)
  }
}

// Joins the pieces of the blocks that shares' edges cut: one CTA per row, of every sequence or, where there are fewer, of every edge (that of a sequence's first
// does the work; the kernel took 32 us by sequences for 256 of them, a quarter of the whole call).  And writes zeros for sequences without tokens, which no
// share has.
__host__ __device__ inline bool joins_by_sequences(int batch, int shares) { return batch < shares || shares == 1; }

__global__ void __launch_bounds__(AMQ_MAX_HEAD_DIM)
cache_attention_join_kernel(const __grid_constant__ AttentionParams p, int block_rows)
{
    grid_dependency_wait();
    const int units = p.c.heads * p.row_blocks, at = blockIdx.x / units, block = blockIdx.x % units, rb = block % p.row_blocks, kv = block / p.row_blocks;
    const int q = blockIdx.y, rho = rb * block_rows + q;
    if (rho >= p.rows) return;
    const int lane = threadIdx.x & 31;
    auto write = [&](int b, float v) {
        const size_t orow = ((size_t)b * p.q_len + rho / p.group) * p.q_heads + kv * p.group + rho % p.group;
        if ((int)threadIdx.x < p.c.d) p.out[orow * p.c.d + threadIdx.x] = v;
    };
    const bool by_sequences = joins_by_sequences(p.batch, p.shares);
    const long long step = by_sequences ? p.batch : p.shares - 1;
    for (long long b0 = at; b0 < p.batch; b0 += 32 * step) {
        const long long e = b0 + lane * step;
        for (uint32_t empty = __ballot_sync(0xffffffffu, e < p.batch && tiles_of(p.c, (int)e) == 0); empty; empty &= empty - 1) write((int)(b0 + (__ffs(empty) - 1) * step), 0.0f);
    }
    const long long total = total_tiles(p);
    const int shares = shares_of(p, total);
    auto edge = [&](int s) { return total * s / shares; };
    long long x = 0;                    // the sequence's place in the line
    int b = at, first;                  // the share that has its first tile
    if (by_sequences) {
        for (int b0 = 0; b0 < b; b0 += 32) {
            const int n = b0 + lane < b ? tiles_of(p.c, b0 + lane) : 0;
            x += (long long)__reduce_add_sync(0xffffffffu, (uint32_t)n & 0xffffu) + ((long long)__reduce_add_sync(0xffffffffu, (uint32_t)n >> 16) << 16);
        }
        if (tiles_of(p.c, b) == 0) return;
        first = (int)(x * shares / total);
        while (edge(first + 1) <= x) ++first;
        while (edge(first) > x) --first;
    } else {
        first = at;
        if (first + 1 >= shares) return;
        b = sequence_at(p, edge(first + 1), &x);
        if (edge(first + 1) == x || edge(first) > x) return;        // (nothing is cut here; cut by an edge before this one)
    }
    const long long end = x + tiles_of(p.c, b);
    int last = first;
    if (edge(first + 1) < end) {
        last = (int)((end - 1) * shares / total);
        while (edge(last + 1) < end) ++last;
        while (edge(last) >= end) --last;
    }
    if (first == last) return;          // (written where it was computed)
    float M = -INFINITY, sum = 0.0f, v = 0.0f;
    auto part = [&](int s) { return (((size_t)s * units + block) * 2 + (s == first ? 1 : 0)) * block_rows + q; };
    for (int s0 = first; s0 <= last; s0 += 32) M = fmaxf(M, s0 + lane <= last ? __ldcg(p.part_ml + part(s0 + lane)).x : -INFINITY);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    const float m_ref = M == -INFINITY ? 0.0f : M;
    for (int s0 = first; s0 <= last; s0 += 32) {
        const float2 ml = s0 + lane <= last ? __ldcg(p.part_ml + part(s0 + lane)) : make_float2(-INFINITY, 0.0f);
        const float f = exp2_approx(ml.x - m_ref);
        sum += ml.y * f;
        const int n = min(32, last - s0 + 1);
#pragma unroll 8
        for (int s = 0; s < n; ++s) v += __ldcg(p.part + part(s0 + s) * AMQ_MAX_HEAD_DIM + threadIdx.x) * __shfl_sync(0xffffffffu, f, s);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    write(b, sum == 0.0f ? 0.0f : v / sum);
}

// all queries' rows in 31 bits, with room for a block behind the last
bool rows_fit(int batch, int q_len, int q_heads)
{
    const long long queries = (long long)batch * q_len;
    return queries <= AMQ_MAX_TOKENS && queries * q_heads <= AMQ_MAX_TOKENS;
}

struct AttentionPlan { int rows, row_tiles, row_blocks, warps, shares; long long blocks; size_t part_bytes, bytes; };

// Up to 1024 tokens a CTA takes a block's whole sequence, with twelve warps (a tile of tokens each or little more) where the CTAs are few: one sequence of
// 300 tokens, 8 heads: 9.2 us, with four warps 9.9.  Else the tiles are dealt out to as many CTAs as fit the GPU, or to fewer of at least 16 tiles.
// Sequences of 1024 tokens, 8 heads, 4 query heads each, whole and in shares: one 16.5 and 17.2 us, 16 17.4 and 22.5, 64 48 and 57, 256 151 and 180;
// of 2048: 8 28.7 and 23, 32 of 512 to 2048 48 and 42.  Up to 2048 tokens whole too where the CTAs are many, so that the GPU evens them out: 256 sequences of up
// to 200 tokens 39 and 67 us, of 1 to 2048 118 and 140 (most of them short) or 177 and 181 (of any length alike), of 2048 279 and 313; three of 2048 among
// 125 short ones are slower, 61 and 53, and with longer ones that grows (8192: 183 and 65).  64 sequences of 1024 to 4096 tokens in equal numbers of
// shares each took 127 us, dealt out 112; one of 65000 tokens 94 and 79.
// Two row tiles to a CTA where rows fill them: 8 rows over 65000 tokens 79 us, 85 with one; 9 rows over 20 x 1500 tokens (3 bits) 47 us, 37 with one.
AttentionPlan attention_plan(int batch, int q_len, int q_heads, int heads, long long max_tokens)
{
    AttentionPlan a{};
    a.rows = q_len * (q_heads / heads);
    const int row_tiles = (a.rows + ROWS - 1) / ROWS;
    const bool whole = max_tokens <= 1024 || (max_tokens <= 2048 && (long long)batch * heads * row_tiles >= 1024);
    a.row_tiles = !whole && row_tiles % 2 == 0 ? 2 : 1;
    const int block = a.row_tiles * ROWS;
    a.row_blocks = (a.rows + block - 1) / block;
    a.blocks = (long long)batch * heads * a.row_blocks;
    a.warps = whole && a.blocks <= 148 ? 12 : 4;
    if (whole) return a;
    const long long units = a.blocks / batch, slots = (a.row_tiles == 1 ? 592 : 296) / units, most = batch * ((max_tokens + TILE - 1) / TILE) / 16;
    const long long shares = most < slots ? most : slots;
    a.shares = (int)(shares < 1 ? 1 : shares);
    const size_t n = (size_t)a.shares * units * 2 * block;
    a.part_bytes = n * AMQ_MAX_HEAD_DIM * 4;
    a.bytes = a.part_bytes + n * sizeof(float2);
    return a;
}

template <int K, int MT, int WARPS>
amq_status launch_attention(const AttentionParams& p, unsigned grid, cudaStream_t st)
{
    constexpr size_t smem = WARPS * (sizeof(Stage<K>) * STAGES + sizeof(Coefficients<K>)), sums = sizeof(float) * WARPS * ROWS * 4 * 33;
    constexpr size_t bytes = smem > sums ? smem : sums;
    auto kernel = cache_attention_kernel<K, MT, WARPS>;
    AMQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    AMQ_CUDA_TRY(launch_kernel(kernel, dim3(grid), dim3(WARPS * 32), bytes, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

template <int K>
amq_status launch_attention_as(const AttentionParams& p, const AttentionPlan& plan, unsigned grid, cudaStream_t st)
{
    if (plan.warps > 4) return launch_attention<K, 1, 12>(p, grid, st);
    return plan.row_tiles == 1 ? launch_attention<K, 1, 4>(p, grid, st) : launch_attention<K, 2, 4>(p, grid, st);
}

}  // namespace
}  // namespace amq

extern "C" {

size_t amq_cache_attention_workspace_bytes(int batch, int q_len, int q_heads, int heads, int d, int max_tokens)
{
    if (batch < 1 || q_len < 1 || q_heads < 1 || heads < 1 || q_heads % heads || d < 1 || d > AMQ_MAX_HEAD_DIM || max_tokens < 1 || !amq::rows_fit(batch, q_len, q_heads)) return 0;
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
    if (!amq::rows_fit(batch, q_len, q_heads)) return AMQ_ERR_UNSUPPORTED;
    if (batch == 0 || q_len == 0) return AMQ_OK;
    if (!q || !out || !lengths || (max_pages > 0 && !table)) return AMQ_ERR_INVALID_ARG;
    if (pages > 0 && (!cache_kcodes || !cache_kcoeffs || !cache_vcodes || !cache_vcoeffs)) return AMQ_ERR_INVALID_ARG;
    if (!amq::aligned16(cache_kcodes) || !amq::aligned16(cache_vcodes)) return AMQ_ERR_ALIGNMENT;
    const amq::AttentionPlan plan = amq::attention_plan(batch, q_len, q_heads, heads, (long long)max_pages * page_size);
    if (plan.blocks > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (plan.bytes) {
        if (!workspace || workspace_bytes < plan.bytes) return AMQ_ERR_WORKSPACE;
        if (!amq::aligned16(workspace)) return AMQ_ERR_ALIGNMENT;
    }
    p.q = q; p.q_batch = q_batch; p.q_token = q_token; p.q_head = q_head;
    p.q_len = q_len; p.q_heads = q_heads; p.group = q_heads / heads; p.scale = scale; p.out = out;
    p.rows = plan.rows; p.row_blocks = plan.row_blocks; p.batch = batch; p.shares = plan.shares;
    const long long grid = plan.shares ? plan.blocks / batch * plan.shares : plan.blocks;
    p.part = static_cast<float*>(workspace);
    p.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + plan.part_bytes);
    p.wide = amq::aligned16(cache_kcoeffs) && amq::aligned16(cache_vcoeffs);
    cudaStream_t st = (cudaStream_t)stream;
    switch (k) {
        case 1: s = amq::launch_attention_as<1>(p, plan, (unsigned)grid, st); break;
        case 2: s = amq::launch_attention_as<2>(p, plan, (unsigned)grid, st); break;
        case 3: s = amq::launch_attention_as<3>(p, plan, (unsigned)grid, st); break;
        default: s = amq::launch_attention_as<4>(p, plan, (unsigned)grid, st); break;
    }
    if (s != AMQ_OK || plan.shares == 0) return s;
    const long long join_blocks = plan.blocks / batch * (amq::joins_by_sequences(batch, plan.shares) ? batch : plan.shares - 1);
    AMQ_CUDA_TRY(amq::launch_kernel(amq::cache_attention_join_kernel, dim3((unsigned)join_blocks, (unsigned)(plan.row_tiles * amq::ROWS)), dim3(AMQ_MAX_HEAD_DIM), 0, st, true, p,
                                    plan.row_tiles * amq::ROWS));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // extern "C"
