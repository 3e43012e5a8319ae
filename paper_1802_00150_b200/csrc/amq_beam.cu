// Beam search on the logits of the output layer (Eq. 6): the choice of the best continuations over beams and vocabulary, and the reordering
// of the states that belong to the chosen beams.
//
// Choice.  score(b, t) = score_b + z_bt - log sum_u exp(z_bu); the `beams` best of all (beam, token) pairs, in the order (score descending, pair
// index ascending).  Within a row the order is that of the logits, so one pass over the logits finds each row's largest and the sum of its
// exponentials together, and only beams x 8 x beams candidates are compared by score, in double: candidates of two beams may lie closer
// than fp32 rounding of a score of -20 (2e-6), those of one beam never change places.
//
// A cluster of eight CTAs takes a batch entry; CTA c reads the eighth c of every beam's row, so any number of beams is balanced, and one entry
// alone still has eight SMs.  A group of 256 threads holds a beam's eighth in registers (in pieces where it has more than 6144 words), one word a
// lane and load, coalesced at any alignment, so that rows of an odd vocabulary cost nothing and the order of a row's sum does not depend
// on where it starts: equal rows get equal sums.  The K-th largest of the maxima of 32 groups of eight lanes is a lower bound of the eighth's K-th
// largest logit, and little more than K logits reach it; those are written down.
#include <cooperative_groups.h>

#include "amq_common.cuh"

namespace amq {
namespace {

namespace cg = cooperative_groups;

constexpr int SLICES = 8;               // CTAs of a cluster
constexpr int THREADS = 256;            // of a group; a CTA has one to four, each with beams of its own
constexpr int WARPS = THREADS / 32;
constexpr int MAX_GROUPS = 4;
constexpr int CAP = 128;                // candidates kept of a beam's slice; where more pass the bound (ties), the slice is searched again

struct SelectParams {
    const float* logits; int ld; int vocab;
    const float* scores; const int32_t* finished; int eos; int beams;
    float* scores_out; int32_t* parents; int32_t* tokens; int32_t* finished_out;
};

// order-preserving maps to unsigned integers (NaN never passes the comparisons in front of them)
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }

// logits larger first, then tokens smaller first: one descending integer order
__device__ __forceinline__ unsigned long long candidate(float v, int token) { return ((unsigned long long)ordered(v) << 32) | (uint32_t)~token; }

struct WarpSum { float m, s; };         // largest logit and sum of exp(z - m) over a warp's share

// shared memory of a CTA: [beams][WARPS] sums, [beams][beams] sorted candidates, then working space
struct SelectSmem {
    WarpSum* sums;
    unsigned long long* best;           // [beams][beams], 0 where there are fewer
    unsigned long long* list;           // [beams][CAP] as found
    int* count;                         // [beams]
    // rank 0: all candidates by score
    double* total;                      // [SLICES * beams * beams]
    int* pair;
};

__host__ __device__ inline size_t select_smem(int beams, SelectSmem* s, void* base)
{
    char* p = static_cast<char*>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* at = p + off; off += (bytes + 15) / 16 * 16; return at; };
    char* sums = take(sizeof(WarpSum) * WARPS * beams);
    char* best = take(8ull * beams * beams);
    char* total = take(8ull * SLICES * beams * beams);      // (the lists are read before the scores are written)
    char* pair = take(4ull * SLICES * beams * beams);
    char* list = take(8ull * CAP * beams);
    char* count = take(4ull * beams);
    if (s) {
        s->sums = reinterpret_cast<WarpSum*>(sums); s->best = reinterpret_cast<unsigned long long*>(best);
        s->list = reinterpret_cast<unsigned long long*>(list);
        s->count = reinterpret_cast<int*>(count); s->total = reinterpret_cast<double*>(total); s->pair = reinterpret_cast<int*>(pair);
    }
    return off;
}

__device__ __forceinline__ uint32_t redux_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }

// (score, pair) a before b
__device__ __forceinline__ bool before(double a, int ai, double b, int bi) { return a > b || (a == b && ai < bi); }

// PT: words of a thread and piece
template <int PT>
__global__ void __cluster_dims__(SLICES, 1, 1) __launch_bounds__(THREADS * MAX_GROUPS)
beam_select_kernel(SelectParams p)
{
    constexpr int CHUNK = THREADS * PT;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float s_score[AMQ_MAX_BEAMS];
    __shared__ int s_done[AMQ_MAX_BEAMS];
    __shared__ double s_lse[AMQ_MAX_BEAMS];
    __shared__ uint32_t s_maxima[MAX_GROUPS][2][32];
    __shared__ double s_cut; __shared__ int s_cut_pair; __shared__ int s_found;
    __shared__ double s_chosen[AMQ_MAX_BEAMS]; __shared__ int s_chosen_pair[AMQ_MAX_BEAMS];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = p.beams, tid = threadIdx.x, nthreads = blockDim.x, lane = tid & 31;
    const int groups = nthreads / THREADS, group = tid / THREADS, at_group = tid % THREADS, warp = at_group >> 5;
    SelectSmem s;
    select_smem(K, &s, smem_raw);
    const int rank = (int)cluster.block_rank(), entry = blockIdx.x / SLICES;
    const int lo = (int)((long long)p.vocab * rank / SLICES), hi = (int)((long long)p.vocab * (rank + 1) / SLICES);
    const size_t row0 = (size_t)entry * K;

    grid_dependency_wait();             // logits, scores and flags may come from the preceding kernel of the stream
    for (int b = tid; b < K; b += nthreads) {
        s_score[b] = p.scores[row0 + b];
        s_done[b] = p.finished ? p.finished[row0 + b] != 0 : 0;
        s.count[b] = 0;
    }
    __syncthreads();

    // a row is read where its candidates can have a score
    auto open = [&](int b) { return !s_done[b] && isfinite(s_score[b]); };
    const int chunks = hi > lo ? (hi - lo + CHUNK - 1) / CHUNK : 0;
    float cur[PT];
    auto load = [&](int b, int c) {
        const float* z = p.logits + (row0 + b) * p.ld;
        const int first = lo + c * CHUNK + at_group;
#pragma unroll
        for (int i = 0; i < PT; ++i) cur[i] = first + i * THREADS < hi ? __ldcg(z + first + i * THREADS) : -INFINITY;
    };
    auto next_open = [&](int b) { while (b < K && !open(b)) b += groups; return b; };

    for (int b = tid; b < K; b += nthreads)
        if (chunks == 0 || !open(b))
            for (int w = 0; w < WARPS; ++w) s.sums[b * WARPS + w] = {-INFINITY, 0.0f};
    int b = chunks ? next_open(group) : K, c = 0, buffer = 0;
    if (b < K) load(b, 0);
    float m = -INFINITY, sum = 0.0f;
    uint32_t bound = 0;                 // below every logit that counts
    while (b < K) {
        // largest and sum of exponentials of this thread's share so far
        float top = cur[0];
#pragma unroll
        for (int i = 1; i < PT; ++i) top = fmaxf(top, cur[i]);
        const uint32_t v = top > -INFINITY ? ordered(top) : 0u;
        uint32_t eight = max(v, __shfl_xor_sync(0xffffffffu, v, 1));
        eight = max(eight, __shfl_xor_sync(0xffffffffu, eight, 2));
        eight = max(eight, __shfl_xor_sync(0xffffffffu, eight, 4));
        if ((lane & 7) == 0) s_maxima[group][buffer][at_group >> 3] = eight;
        const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.0f : m_new;
        sum *= __expf(m - ref);
#pragma unroll
        for (int i = 0; i < PT; ++i) sum += __expf(cur[i] - ref);
        m = m_new;
        asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "n"(THREADS) : "memory");
        // (the two buffers in turn: who writes one again has passed the barrier behind everybody's reading of it)
        uint32_t left = s_maxima[group][buffer][lane];
        buffer ^= 1;
        if (redux_max(left) > bound) {
            uint32_t kth = 0;
            for (int r = 0; r < K; ++r) {
                kth = redux_max(left);
                const uint32_t has = __ballot_sync(0xffffffffu, left == kth);
                if (lane == __ffs(has) - 1) left = 0u;
            }
            bound = max(bound, kth);
        }
        if (v && v >= bound) {
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                if (cur[i] > -INFINITY && ordered(cur[i]) >= bound) {
                    const int to = atomicAdd(&s.count[b], 1);
                    if (to < CAP) s.list[b * CAP + to] = candidate(cur[i], lo + c * CHUNK + at_group + i * THREADS);
                }
            }
        }
        int nb = b, nc = c + 1;
        if (nc == chunks) { nc = 0; nb = next_open(b + groups); }
        if (nb < K) load(nb, nc);
        if (nb != b) {                  // the row is through: the warp's share of its sum
            const uint32_t wm = redux_max(m > -INFINITY ? ordered(m) : 0u);
            const float M = wm ? from_ordered(wm) : -INFINITY;
            float t = sum * __expf(m - (wm ? M : 0.0f));        // (nothing but -inf: 0)
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
            if (lane == 0) s.sums[b * WARPS + warp] = {M, t};
            m = -INFINITY; sum = 0.0f; bound = 0;
        }
        b = nb; c = nc;
    }
    __syncthreads();

    // the K best of each beam's slice, in order: a candidate's place is the number of candidates before it
    for (int q = tid >> 5; q < K; q += nthreads >> 5) {
        const int n = s.count[q];
        unsigned long long* best = s.best + (size_t)q * K;
        if (n <= CAP) {
            for (int r = (n < K ? n : K) + lane; r < K; r += 32) best[r] = 0;
            for (int i = lane; i < n; i += 32) {
                const unsigned long long mine = s.list[q * CAP + i];
                int place = 0;
                for (int j = 0; j < n; ++j) place += s.list[q * CAP + j] > mine;
                if (place < K) best[place] = mine;
            }
        } else {                        // more ties than the list holds: one search of the slice for every place
            const float* z = p.logits + (row0 + q) * p.ld;
            unsigned long long last = ~0ull;
            for (int r = 0; r < K; ++r) {
                unsigned long long top = 0;
                for (int t = lo + lane; t < hi; t += 32) {
                    const float x = __ldcg(z + t);
                    if (!(x > -INFINITY)) continue;
                    const unsigned long long k = candidate(x, t);
                    if (k < last && k > top) top = k;
                }
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) {
                    const unsigned long long o = __shfl_xor_sync(0xffffffffu, top, off);
                    if (o > top) top = o;
                }
                if (lane == 0) best[r] = top;
                last = top;
            }
        }
    }
    cluster.sync();
    if (rank == 0) {
        // log-sum-exp of each row, from the 64 warps' shares, in double
        for (int q = tid >> 5; q < K; q += nthreads >> 5) {
            float wm[2], ws[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int w = lane + 32 * h;
                const WarpSum* there = cluster.map_shared_rank(s.sums, w / WARPS);
                wm[h] = there[q * WARPS + w % WARPS].m; ws[h] = there[q * WARPS + w % WARPS].s;
            }
            float M = fmaxf(wm[0], wm[1]);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
            double t = 0.0;
            if (isfinite(M)) t = (double)ws[0] * exp((double)wm[0] - M) + (double)ws[1] * exp((double)wm[1] - M);
            else t = NAN;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
            if (lane == 0) s_lse[q] = (double)M + log(t);
        }
        if (tid == 0) { s_found = 0; s_cut = -INFINITY; s_cut_pair = 0x7fffffff; }
        __syncthreads();
        // every candidate's score; a beam's lists lie one behind the other, [beam][slice][place]
        const int all = K * SLICES * K;
        for (int i = tid; i < all; i += nthreads) {
            const int q = i / (SLICES * K), slice = i / K % SLICES, r = i % K;
            double total = -INFINITY;
            int pair = 0x7fffffff;
            if (open(q)) {
                const unsigned long long k = cluster.map_shared_rank(s.best, slice)[q * K + r];
                const double lse = s_lse[q];
                if (k && isfinite(lse)) {
                    total = (double)s_score[q] + ((double)from_ordered((uint32_t)(k >> 32)) - lse);
                    pair = q * p.vocab + (int)~(uint32_t)k;
                }
            } else if (s_done[q] && slice == 0 && r == 0 && isfinite(s_score[q])) {
                total = (double)s_score[q];
                pair = q * p.vocab + p.eos;
            }
            s.total[i] = total; s.pair[i] = pair;
        }
    }
    cluster.sync();                     // nobody's shared memory is read any more
    if (rank != 0) return;

    // The K-th best of the lists' heads bounds what can be chosen: at most K lists reach it.  (Heads without a candidate are all alike and last.)
    const int heads = K * SLICES;
    for (int i = tid; i < heads; i += nthreads) {
        const double mine = s.total[i * K];
        const int pair = s.pair[i * K];
        if (pair == 0x7fffffff) continue;
        int place = 0;
        for (int j = 0; j < heads; ++j) place += before(s.total[j * K], s.pair[j * K], mine, pair);
        if (place == K - 1) { s_cut = mine; s_cut_pair = pair; }
    }
    __syncthreads();
    // candidates at or before the bound, written down (over the lists of this CTA, which have been read)
    double* kept = reinterpret_cast<double*>(s.best);                       // [K * K] doubles
    int* kept_pair = reinterpret_cast<int*>(s.list);                        // [K * CAP * 2] words: K * K fit
    for (int i = tid; i < K * SLICES * K; i += nthreads) {
        const int pair = s.pair[i];
        if (pair == 0x7fffffff || before(s_cut, s_cut_pair, s.total[i], pair)) continue;
        const int at = atomicAdd(&s_found, 1);
        kept[at] = s.total[i]; kept_pair[at] = pair;
    }
    __syncthreads();
    const int found = s_found;
    for (int i = tid; i < found; i += nthreads) {
        int place = 0;
        for (int j = 0; j < found; ++j) place += before(kept[j], kept_pair[j], kept[i], kept_pair[i]);
        if (place < K) { s_chosen[place] = kept[i]; s_chosen_pair[place] = kept_pair[i]; }
    }
    __syncthreads();
    if (tid == 0 && found < K) {        // fewer candidates than beams: the first pairs that are none, with a score of -inf
        int pair = 0;
        for (int r = found; r < K; ++r, ++pair) {
            for (bool taken = true; taken;) {
                taken = false;
                for (int j = 0; j < found; ++j) taken |= s_chosen_pair[j] == pair;
                if (taken) ++pair;
            }
            s_chosen[r] = -INFINITY; s_chosen_pair[r] = pair;
        }
    }
    __syncthreads();
    if (tid < K) {
        const int pair = s_chosen_pair[tid], parent = pair / p.vocab, token = pair - parent * p.vocab;
        p.scores_out[row0 + tid] = (float)s_chosen[tid];
        p.parents[row0 + tid] = parent;
        p.tokens[row0 + tid] = token;
        if (p.finished_out) p.finished_out[row0 + tid] = (s_done[parent] || token == p.eos) ? 1 : 0;
    }
}

template <int PT>
amq_status launch_select_as(const SelectParams& p, int batch, int groups, cudaStream_t st)
{
    const size_t smem = select_smem(p.beams, nullptr, nullptr);
    AMQ_CUDA_TRY(cudaFuncSetAttribute(beam_select_kernel<PT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    AMQ_CUDA_TRY(launch_kernel(beam_select_kernel<PT>, dim3((unsigned)(batch * SLICES)), dim3((unsigned)(THREADS * groups)), smem, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

amq_status launch_select(const SelectParams& p, int batch, cudaStream_t st)
{
    // beams at a time: as many as leave the CTAs of all entries on the GPU at once
    int groups = batch * SLICES <= 148 ? MAX_GROUPS : batch * SLICES <= 296 ? 2 : 1;
    if (groups > p.beams) groups = p.beams;
    const int slice = (p.vocab + SLICES - 1) / SLICES, pieces = (slice + THREADS * 24 - 1) / (THREADS * 24);
    const int words = ((slice + pieces - 1) / pieces + THREADS - 1) / THREADS;
    if (words <= 2) return launch_select_as<2>(p, batch, groups, st);
    if (words <= 5) return launch_select_as<5>(p, batch, groups, st);
    if (words <= 8) return launch_select_as<8>(p, batch, groups, st);
    if (words <= 12) return launch_select_as<12>(p, batch, groups, st);
    if (words <= 16) return launch_select_as<16>(p, batch, groups, st);
    return launch_select_as<24>(p, batch, groups, st);
}

// ---- reordering ------------------------------------------------------------------------------------------------------

struct ReorderParams {
    const char* src[AMQ_MAX_STATES]; char* dst[AMQ_MAX_STATES];
    long long src_stride[AMQ_MAX_STATES], dst_stride[AMQ_MAX_STATES];
    int columns[AMQ_MAX_STATES];        // words of type V in a row
    const int32_t* parents;
    int batch, beams;
};

// A thread owns one column of a batch entry across all its beams: it reads the parents' values first and writes after, so the states may be
// reordered in place without a second copy.  K: registers for the beams.
template <typename V, int K>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(const __grid_constant__ ReorderParams p)
{
    grid_dependency_wait();
    const int st = blockIdx.y, columns = p.columns[st];
    const long long all = (long long)p.batch * columns;
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < all; at += (long long)gridDim.x * 256) {
        const int entry = (int)(at / columns), column = (int)(at - (long long)entry * columns);
        const long long row0 = (long long)entry * p.beams;
        const char* src = p.src[st] + row0 * p.src_stride[st] + (long long)column * sizeof(V);
        char* dst = p.dst[st] + row0 * p.dst_stride[st] + (long long)column * sizeof(V);
        V v[K];
        int parent[K];
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (b < p.beams) {
                const int q = p.parents[row0 + b];
                parent[b] = q < 0 ? 0 : q < p.beams ? q : p.beams - 1;
            }
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (b < p.beams) v[b] = *reinterpret_cast<const V*>(src + parent[b] * p.src_stride[st]);
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (b < p.beams && (parent[b] != b || src != dst)) *reinterpret_cast<V*>(dst + b * p.dst_stride[st]) = v[b];
    }
}

template <typename V>
amq_status launch_reorder(const ReorderParams& p, int count, cudaStream_t st)
{
    auto kernel = p.beams <= 4 ? beam_reorder_kernel<V, 4> : p.beams <= 8 ? beam_reorder_kernel<V, 8>
                : p.beams <= 16 ? beam_reorder_kernel<V, 16> : beam_reorder_kernel<V, 32>;
    long long most = 0;
    for (int i = 0; i < count; ++i) if (p.columns[i] > most) most = p.columns[i];
    long long blocks = (most * p.batch + 255) / 256;
    if (blocks > 1 << 20) blocks = 1 << 20;
    AMQ_CUDA_TRY(launch_kernel(kernel, dim3((unsigned)blocks, (unsigned)count), dim3(256), 0, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // namespace
}  // namespace amq

extern "C" {

amq_status amq_beam_select(const float* logits, int ld, int vocab, const float* scores, const int32_t* finished, int eos, int batch, int beams,
                           float* scores_out, int32_t* parents, int32_t* tokens, int32_t* finished_out, void* stream)
{
    if (vocab < 1 || ld < vocab || batch < 0 || beams < 1 || eos < -1 || eos >= vocab || (finished && eos < 0)) return AMQ_ERR_INVALID_ARG;
    if (beams > AMQ_MAX_BEAMS || (long long)beams * vocab > 0x7ffffffell || (long long)batch * amq::SLICES > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
    if (batch == 0) return AMQ_OK;
    if (!logits || !scores || !scores_out || !parents || !tokens) return AMQ_ERR_INVALID_ARG;
    amq::SelectParams p{logits, ld, vocab, scores, finished, eos, beams, scores_out, parents, tokens, finished_out};
    return amq::launch_select(p, batch, (cudaStream_t)stream);
}

amq_status amq_beam_reorder(const void* const* src, void* const* dst, const size_t* row_bytes, const size_t* src_stride, const size_t* dst_stride,
                            int count, const int32_t* parents, int batch, int beams, void* stream)
{
    if (count < 0 || batch < 0 || beams < 1) return AMQ_ERR_INVALID_ARG;
    if (count > AMQ_MAX_STATES || beams > AMQ_MAX_BEAMS) return AMQ_ERR_UNSUPPORTED;
    if (count == 0 || batch == 0) return AMQ_OK;
    if (!src || !dst || !row_bytes || !src_stride || !dst_stride || !parents) return AMQ_ERR_INVALID_ARG;
    amq::ReorderParams p{};
    p.parents = parents; p.batch = batch; p.beams = beams;
    bool wide = true;                   // every row of every state in 16-byte words
    for (int i = 0; i < count; ++i) {
        if (src_stride[i] < row_bytes[i] || dst_stride[i] < row_bytes[i] || (src[i] == dst[i] && src_stride[i] != dst_stride[i])) return AMQ_ERR_INVALID_ARG;
        if (row_bytes[i] && (!src[i] || !dst[i])) return AMQ_ERR_INVALID_ARG;
        if (row_bytes[i] / 4 > 0x7fffffffu) return AMQ_ERR_UNSUPPORTED;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(src[i]) | reinterpret_cast<uintptr_t>(dst[i]) | row_bytes[i] | src_stride[i] | dst_stride[i];
        if (bits & 3) return AMQ_ERR_ALIGNMENT;
        if (bits & 15) wide = false;
        p.src[i] = static_cast<const char*>(src[i]); p.dst[i] = static_cast<char*>(dst[i]);
        p.src_stride[i] = (long long)src_stride[i]; p.dst_stride[i] = (long long)dst_stride[i];
    }
    long long most = 0;
    for (int i = 0; i < count; ++i) {
        p.columns[i] = (int)(row_bytes[i] / (wide ? 16 : 4));
        if (p.columns[i] > most) most = p.columns[i];
    }
    if (most == 0) return AMQ_OK;
    return wide ? amq::launch_reorder<uint4>(p, count, (cudaStream_t)stream) : amq::launch_reorder<uint32_t>(p, count, (cudaStream_t)stream);
}

}  // extern "C"
