// Beam search on the logits of the output layer (Eq. 6): the choice of the best continuations over beams and vocabulary, and the reordering
// of the states that belong to the chosen beams.
//
// Choice.  score(b, t) = score_b + z_bt - log sum_u exp(z_bu); the `beams` best of all (beam, token) pairs, in the order (score descending, pair
// index ascending).  Within a row the order is that of the logits (also where different logits round to one score), so one pass over the logits finds each
// row's largest and the sum of its exponentials together, and only beams x 8 x beams candidates are compared by score, in double: candidates
// of two beams may lie closer than fp32 rounding of a score of -20 (2e-6).
//
// A cluster of eight or four CTAs takes a batch entry; CTA c reads the share c of every beam's row, so any number of beams is balanced, and one entry
// alone still has eight SMs.  A group of 128 or 256 threads takes a beam's share in pieces of up to 24 words a thread, with up to twelve the next piece on its
// way while one is worked on: one word a lane and load, coalesced at any alignment, so that rows of an odd vocabulary cost nothing and the order of a row's
// sum does not depend on where it starts: equal rows get equal sums.  A lower bound of the share's K-th largest logit comes from the maxima of 32 or 64 groups
// of threads, and little more than K logits reach it; those are written down, sorted by a warp, and go to the first CTA's shared memory, which
// joins them by score.
// Bound by instructions and barriers, 17 instructions for a lane and logit at 21 logits a thread and piece: load, maximum, exponential, sum, and some 240 a warp and
// piece for the bound, the candidates and the sums.  64 entries, 8 beams, 42000 tokens: 26.7 us, 3.2 TB/s (a CTA to an entry, a pass for the sum and
// one for each beam: 149 us); one entry, 5 beams, 9999 tokens: 7.3 us, a chain of two barriers, the cluster's exchange and the join.
#include <cooperative_groups.h>

#include <type_traits>

#include "amq_common.cuh"
#include "amq_pairs.cuh"

namespace amq {
namespace {

namespace cg = cooperative_groups;

constexpr int MAX_THREADS = 1024;       // of a CTA: groups of 128 or 256 threads, each with beams of its own
constexpr int MAX_GROUPS = 8, MAX_WARPS = 8;        // groups, warps of a group
constexpr int CAP = 256;                // candidates kept of a beam's slice; where more pass the bound (ties), the slice is searched again
constexpr int MAXIMA = 64;

struct SelectParams {
    const float* logits; int ld; int vocab;
    const float* scores; const int32_t* finished; int eos; int beams;
    float* scores_out; int32_t* parents; int32_t* tokens; int32_t* finished_out;
};

// order-preserving maps to unsigned integers (NaN never passes the comparisons in front of them); -0 is 0
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr uint32_t LOWEST = 0x00800000u;       // of -FLT_MAX
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }

// logits larger first, then tokens smaller first: one descending integer order
__device__ __forceinline__ unsigned long long candidate(float v, int token) { return ((unsigned long long)ordered(v) << 32) | (uint32_t)~token; }

// one instruction, within 2^-22 of itself: less than the roundings of a piece's sum; twice as exact, a double's worth of work on 512 x 42000 logits would take longer
// than all the rest
__device__ __forceinline__ float exp2_ftz(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
constexpr float LOG2E = 1.44269504f;

// Sums of exp(z) as s exp(m), m = the largest logit: the exponents (z - m) LOG2E are two roundings each, relative to themselves, and no finite logit is too
// large for them (m LOG2E is, from 2.4e38 on).
struct WarpSum { float m, s; };
__device__ __forceinline__ float exp_from(float z, float m) { return exp2_ftz((z - m) * LOG2E); }

// shared memory of a CTA.  What the others send lies in the first CTA's.
struct SelectSmem {
    WarpSum* sums;                      // [beams][slices][warps of a group], from every CTA
    unsigned long long* best;           // [beams][slices][beams], from every CTA: sorted candidates, 0 where there are fewer
    unsigned long long* list;           // [beams][CAP] as found
};

__host__ __device__ inline size_t select_smem(int slices, int beams, SelectSmem* s, void* base)
{
    char* p = static_cast<char*>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* at = p + off; off += (bytes + 15) / 16 * 16; return at; };
    char* sums = take(sizeof(WarpSum) * slices * MAX_WARPS * beams);
    char* best = take(8ull * slices * beams * beams);
    char* list = take(8ull * CAP * beams);
    if (s) {
        s->sums = reinterpret_cast<WarpSum*>(sums); s->best = reinterpret_cast<unsigned long long*>(best);
        s->list = reinterpret_cast<unsigned long long*>(list);
    }
    return off;
}

__device__ __forceinline__ uint32_t redux_max(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }

// doubles in the order of unsigned integers (finite ones)
__device__ __forceinline__ unsigned long long ordered(double v)
{
    const unsigned long long u = (unsigned long long)__double_as_longlong(v);
    return u ^ ((unsigned long long)((long long)u >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ double from_ordered(unsigned long long o)
{
    return __longlong_as_double((long long)(o ^ ((o >> 63) ? 0x8000000000000000ull : 0xffffffffffffffffull)));
}

// the 32 best of `kept`, in descending order over a warp's lanes, and 32 others in any, in descending order: a bitonic sort of those, ascending, and a merge
__device__ __forceinline__ unsigned long long best_of(unsigned long long kept, unsigned long long other)
{
    const int lane = threadIdx.x & 31;
    auto exchange = [&](unsigned long long v, int stride, bool larger) {
        const unsigned long long o = __shfl_xor_sync(0xffffffffu, v, stride);
        return (o > v) == larger ? o : v;
    };
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int stride = size >> 1; stride > 0; stride >>= 1) other = exchange(other, stride, ((lane & stride) != 0) == ((lane & size & 31) == 0));
    if (other > kept) kept = other;
#pragma unroll
    for (int stride = 16; stride > 0; stride >>= 1) kept = exchange(kept, stride, (lane & stride) == 0);
    return kept;
}

struct Choice { unsigned long long score; int pair; };       // score 0: none

// One warp joins the sorted lists (one for each beam and slice, SLICES a beam): LISTS of them a lane, and beam after beam of the result the best of their heads: by
// score; equal scores by beam, of one beam by logit (different logits may give one score, of a beam far below the others: a step of a double of -1e9 is 1e-7), then by
// token.  `score_of(list, place)`, `logit_of(list, place)` in the order of integers.  Returns how many there were; lane 0 has written them down.
template <int SLICES, int LISTS, typename F, typename G>
__device__ __forceinline__ int join_lists(int K, int lists, F&& score_of, G&& logit_of, double* chosen, int* chosen_pair)
{
    static_assert(32 % SLICES == 0, "a lane's lists are of different beams, the first of them of the smallest");
    const int lane = threadIdx.x & 31;
    Choice head[LISTS];
    int place[LISTS];
#pragma unroll
    for (int x = 0; x < LISTS; ++x) {
        place[x] = 0;
        head[x] = lane + 32 * x < lists ? score_of(lane + 32 * x, 0) : Choice{0ull, 0};
    }
    for (int r = 0; r < K; ++r) {
        Choice best = head[0];
        int from = 0;
#pragma unroll
        for (int x = 1; x < LISTS; ++x)
            if (head[x].score > best.score) { best = head[x]; from = x; }
        const uint32_t hi = redux_max((uint32_t)(best.score >> 32));
        if (hi == 0u) return r;                     // (a finite score's high word is not 0)
        const uint32_t lo = redux_max((uint32_t)(best.score >> 32) == hi ? (uint32_t)best.score : 0u);
        uint32_t top = __ballot_sync(0xffffffffu, best.score == (((unsigned long long)hi << 32) | lo));
        if (top & (top - 1)) {
            auto among = [&](uint32_t v) {          // the lanes of `top` with the smallest value
                const bool in = top >> lane & 1;
                const uint32_t least = __reduce_min_sync(0xffffffffu, in ? v : 0xffffffffu);       // (all lanes, in front of any condition)
                top = __ballot_sync(0xffffffffu, in && v == least);
            };
            among((uint32_t)((lane + 32 * from) / SLICES));
            int at = place[0];
#pragma unroll
            for (int x = 1; x < LISTS; ++x) at = x == from ? place[x] : at;
            among(top >> lane & 1 ? ~logit_of(lane + 32 * from, at) : 0xffffffffu);
            among((uint32_t)best.pair);             // (pairs are distinct: one lane)
        }
        const int winner = __ffs(top) - 1;
        const int pair = __shfl_sync(0xffffffffu, best.pair, winner);
        if (lane == 0) { chosen[r] = from_ordered(((unsigned long long)hi << 32) | lo); chosen_pair[r] = pair; }
        if (lane == winner) {
#pragma unroll
            for (int x = 0; x < LISTS; ++x)
                if (x == from) head[x] = ++place[x] < K ? score_of(lane + 32 * x, place[x]) : Choice{0ull, 0};
        }
    }
    return K;
}

// SLICES: CTAs of a cluster; THREADS: of a group; PT: words of a thread and piece
template <int SLICES, int THREADS, int PT>
__global__ void __cluster_dims__(SLICES, 1, 1) __launch_bounds__(MAX_THREADS, 1)
beam_select_kernel(SelectParams p)
{
    constexpr int CHUNK = THREADS * PT, WARPS = THREADS / 32;
    constexpr int SURE = PT <= 2 ? 0 : PT == 5 ? 2 : PT == 8 ? 5 : PT == 10 ? 8 : PT == 12 ? 10 : PT == 16 ? 12 : PT == 21 ? 16 : 21;      // (the size below)
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float s_score[AMQ_MAX_BEAMS];
    __shared__ int s_done[AMQ_MAX_BEAMS];
    __shared__ float s_top[AMQ_MAX_BEAMS]; __shared__ double s_log[AMQ_MAX_BEAMS];       // a row's largest logit, and the logarithm of its sum relative to that
    __shared__ uint32_t s_maxima[MAX_GROUPS][2][MAXIMA];
    __shared__ int s_count[AMQ_MAX_BEAMS]; __shared__ uint32_t s_bound[AMQ_MAX_BEAMS];
    __shared__ int s_found;
    __shared__ double s_chosen[AMQ_MAX_BEAMS]; __shared__ int s_chosen_pair[AMQ_MAX_BEAMS];
    cg::cluster_group cluster = cg::this_cluster();
    const int K = p.beams, tid = threadIdx.x, nthreads = blockDim.x, lane = tid & 31;
    const int groups = nthreads / THREADS, group = tid / THREADS, at_group = tid % THREADS, warp = at_group >> 5;
    SelectSmem s;
    select_smem(SLICES, K, &s, smem_raw);
    const int rank = (int)cluster.block_rank(), entry = blockIdx.x / SLICES;
    const int lo = (int)((long long)p.vocab * rank / SLICES), hi = (int)((long long)p.vocab * (rank + 1) / SLICES);
    const size_t row0 = (size_t)entry * K;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");        // (the first CTA runs before anything is sent to it: waited for below)

    grid_dependency_wait();             // logits, scores and flags may come from the preceding kernel of the stream
    const int chunks = hi > lo ? (hi - lo + CHUNK - 1) / CHUNK : 0;
    constexpr bool AHEAD = PT <= 12;    // a second piece in registers, fetched while one is worked on; with longer ones the SM's other CTAs have to do
    float cur[PT], nxt[AHEAD ? PT : 1];
    auto load = [&](float (&v)[PT], int b, int c) {
        const int left = hi - lo - c * CHUNK;       // words from this piece on (a place behind the share may lie behind 2^31; what is left never does)
        const float* z = p.logits + (row0 + b) * p.ld + (size_t)(lo + c * CHUNK) + at_group;
        if (left >= CHUNK) {
#pragma unroll
            for (int i = 0; i < PT; ++i) v[i] = __ldcg(z + i * THREADS);
        } else if (left >= SURE * THREADS) {        // (a row's only piece, as a rule: its first words need no comparison)
#pragma unroll
            for (int i = 0; i < PT; ++i) v[i] = i < SURE || at_group + i * THREADS < left ? __ldcg(z + i * THREADS) : -INFINITY;
        } else {
#pragma unroll
            for (int i = 0; i < PT; ++i) v[i] = at_group + i * THREADS < left ? __ldcg(z + i * THREADS) : -INFINITY;
        }
    };
    if (chunks && group < K) load(cur, group, 0);           // (whether it counts is not known yet)
    for (int b = tid; b < K; b += nthreads) {
        s_score[b] = p.scores[row0 + b];
        s_done[b] = p.finished ? p.finished[row0 + b] != 0 : 0;
        s_count[b] = 0;
    }
    __syncthreads();

    // a row is looked at where its candidates can have a score
    auto open = [&](int b) { return !s_done[b] && isfinite(s_score[b]); };
    auto next_open = [&](int b) { while (b < K && !open(b)) b += groups; return b; };
    WarpSum* const sums_there = cluster.map_shared_rank(s.sums, 0) + rank * WARPS;
    unsigned long long* const best_there = cluster.map_shared_rank(s.best, 0) + (size_t)rank * K;

    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (chunks == 0) {
        for (int i = tid; i < K * WARPS; i += nthreads) sums_there[i / WARPS * SLICES * WARPS + i % WARPS] = {-INFINITY, 0.0f};
        for (int i = tid; i < K * K; i += nthreads) best_there[(size_t)(i / K) * SLICES * K + i % K] = 0;
    }

    int b = chunks ? next_open(group) : K, c = 0, buffer = 0;
    if (b < K && b != group) load(cur, b, 0);
    float m = -INFINITY;
    double sum = 0.0;                   // (over pieces: in fp32 many equal terms of a long row would all be rounded one way, 4e-6 for 300000 tokens)
    uint32_t bound = 0, highest = 0;    // below every logit that counts; this thread's largest of the row so far
    // one piece, and the next one's loads
    auto step = [&](float (&now)[PT], auto& next) {
        int nb = b, nc = c + 1;
        if (nc == chunks) { nc = 0; nb = next_open(b + groups); }
        if constexpr (AHEAD) { if (nb < K) load(next, nb, nc); }
        // largest and sum of exponentials of this thread's share so far
        float top = now[0];
#pragma unroll
        for (int i = 1; i < PT; ++i) top = fmaxf(top, now[i]);
        const uint32_t v = top > -INFINITY ? ordered(top) : 0u;
        highest = max(highest, v);
        // (a row's second piece goes by the first one's bound: another would rarely spare it much)
        if (c != 1) {
            uint32_t of_some = max(highest, __shfl_xor_sync(0xffffffffu, highest, 1));
            if (THREADS == 256) of_some = max(of_some, __shfl_xor_sync(0xffffffffu, of_some, 2));
            if (K <= 8) {               // 32 maxima, else 64
                of_some = max(of_some, __shfl_xor_sync(0xffffffffu, of_some, THREADS / 64));
                if ((lane & (THREADS / 32 - 1)) == 0) s_maxima[group][buffer][at_group / (THREADS / 32)] = of_some;
            } else if ((lane & (THREADS / 64 - 1)) == 0) {
                s_maxima[group][buffer][at_group / (THREADS / 64)] = of_some;
            }
        }
        const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.0f : m_new;
        {
            float even = 0.0f, odd = 0.0f;          // of the piece, 12 words each
            const f32x2 less = pack2(-ref, -ref), scale = pack2(LOG2E, LOG2E);
#pragma unroll
            for (int i = 0; i + 1 < PT; i += 2) {
                float e0, e1;
                unpack2(mul2(add2(pack2(now[i], now[i + 1]), less), scale), e0, e1);
                even += exp2_ftz(e0);
                odd += exp2_ftz(e1);
            }
            if (PT & 1) even += exp_from(now[PT - 1], ref);
            sum = fma(sum, (double)exp_from(m, ref), (double)(even + odd));
        }
        m = m_new;
        if (c != 1) {
            asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "n"(THREADS) : "memory");
            // The bound, one that K threads' largest logits reach.  Up to four beams the smallest of four maxima (of a quarter of the threads; 8 logits
            // reach it on average, 50 once in a million), up to eight the smallest of four second largest, of eight maxima each (14; one by one, the
            // K-th largest of 32 took 32.5 us where this took 28.9), else a value that K to 5 K / 4 of 64 maxima reach, by bisection.  The two
            // buffers in turn: who writes one again has passed the barrier behind everybody's reading of it.
            uint32_t left = s_maxima[group][buffer][lane];
            if (K <= 4) {
                left = max(left, __shfl_xor_sync(0xffffffffu, left, 4));
                left = max(left, __shfl_xor_sync(0xffffffffu, left, 8));
                left = max(left, __shfl_xor_sync(0xffffffffu, left, 16));
                bound = max(bound, __reduce_min_sync(0xffffffffu, left));
            } else if (K <= 8) {
                uint32_t second = 0;
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) {
                    const uint32_t l2 = __shfl_xor_sync(0xffffffffu, left, off), s2 = off == 4 ? 0u : __shfl_xor_sync(0xffffffffu, second, off);
                    second = max(min(left, l2), off == 4 ? 0u : max(second, s2));
                    left = max(left, l2);
                }
                bound = max(bound, __reduce_min_sync(0xffffffffu, second));
            } else {
                const uint32_t right = s_maxima[group][buffer][32 + lane];
                // K reach `from` (or it is the bound already), fewer `to` + 1
                uint32_t from = max(bound, __reduce_min_sync(0xffffffffu, min(left, right))), to = redux_max(max(left, right));
                while (from < to) {
                    const uint32_t mid = from + (to - from + 1) / 2;
                    const int n = __popc(__ballot_sync(0xffffffffu, left >= mid)) + __popc(__ballot_sync(0xffffffffu, right >= mid));
                    if (n >= K) from = mid;
                    else to = mid - 1;
                    if (n >= K && n <= K + K / 4) break;
                }
                bound = from;
            }
            buffer ^= 1;
        }
        if (v && v >= bound) {
            // (a bound below every finite logit's is none: everything but -inf.  The bisection may end there, among the places of -inf and NaN, where a
            // slice has few logits above the type's lowest value)
            const float least = from_ordered(max(bound, LOWEST));
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                if (now[i] >= least) {
                    const int to = atomicAdd(&s_count[b], 1);
                    if (to < CAP) s.list[b * CAP + to] = candidate(now[i], lo + c * CHUNK + at_group + i * THREADS);
                }
            }
        }
        if constexpr (!AHEAD) { if (nb < K) load(now, nb, nc); }
        if (nb != b) {                  // the row is through: the warp's share of its sum
            const uint32_t wm = redux_max(m > -INFINITY ? ordered(m) : 0u);
            const float M = wm ? from_ordered(wm) : -INFINITY;
            float t = (float)sum * exp_from(m, wm ? M : 0.0f);           // (nothing but -inf: 0)
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
            if (lane == 0) sums_there[b * SLICES * WARPS + warp] = {M, t};
            if (at_group == 0) s_bound[b] = bound;
            m = -INFINITY; sum = 0.0; bound = 0; highest = 0;
        }
        b = nb; c = nc;
    };
    while (b < K) {
        step(cur, nxt);
        if constexpr (AHEAD) { if (b < K) step(nxt, cur); }
    }
    __syncthreads();

    // the K best of each beam's slice, in order, a warp a beam
    for (int q = tid >> 5; q < K; q += nthreads >> 5) {
        const int n = s_count[q];
        const unsigned long long* list = s.list + q * CAP;
        unsigned long long* best = best_there + (size_t)q * SLICES * K;
        if (n <= 32) {                  // (as a rule: a candidate's place is the number of candidates before it)
            const unsigned long long mine = lane < n ? list[lane] : 0ull;
            int before = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) before += __shfl_sync(0xffffffffu, mine, j) > mine;
            if (before < K && mine) best[before] = mine;
            if (lane >= n && lane < K) best[lane] = 0;
        } else if (n <= CAP) {
            unsigned long long kept = 0;
            for (int i = lane; i - lane < n; i += 32) kept = best_of(kept, i < n ? list[i] : 0ull);
            if (lane < K) best[lane] = kept;
        } else {                        // more ties than the list holds: the slice once more, past the best so far, a place of which each lane keeps
            const float* z = p.logits + (row0 + q) * p.ld + lo;
            const uint32_t least = s_bound[q];
            unsigned long long kept = 0;
            for (int t0 = 0; t0 < hi - lo; t0 += 128) {             // (a share is a quarter of the vocabulary at most)
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = t0 + 32 * i + lane < hi - lo ? __ldcg(z + t0 + 32 * i + lane) : -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned long long k = x[i] > -INFINITY && ordered(x[i]) >= least ? candidate(x[i], lo + t0 + 32 * i + lane) : 0ull;
                    uint32_t above = __ballot_sync(0xffffffffu, k > __shfl_sync(0xffffffffu, kept, K - 1));
                    for (; above; above &= above - 1) {
                        const unsigned long long one = __shfl_sync(0xffffffffu, k, __ffs(above) - 1), up = __shfl_up_sync(0xffffffffu, kept, 1);
                        const int place = __popc(__ballot_sync(0xffffffffu, kept > one));
                        kept = lane < place ? kept : lane == place ? one : up;
                    }
                }
            }
            if (lane < K) best[lane] = kept;
        }
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    if (rank != 0) return;              // (nobody reads another CTA's shared memory, and the first one stays)
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");

    // log-sum-exp of each row, from the warps' shares, summed in double
    for (int q = tid >> 5; q < K; q += nthreads >> 5) {
        if (!open(q)) continue;
        constexpr int SHARES = SLICES * WARPS / 32;
        WarpSum w[SHARES];
        float M = -INFINITY;
#pragma unroll
        for (int x = 0; x < SHARES; ++x) { w[x] = s.sums[q * SLICES * WARPS + 32 * x + lane]; M = fmaxf(M, w[x].m); }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
        double t = isfinite(M) ? 0.0 : (double)NAN;
#pragma unroll
        for (int x = 0; x < SHARES; ++x) t += (double)(w[x].s * exp2f((w[x].m - M) * LOG2E));
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
        if (lane == 0) { s_top[q] = M; s_log[q] = log(t); }
    }
    __syncthreads();
    if (tid < 32) {
        // a beam's lists lie one behind the other, [beam][slice][place]; a beam that has ended has one candidate
        auto score_of = [&](int list, int place) {
            const int q = list / SLICES;
            if (open(q)) {
                const unsigned long long k = s.best[(size_t)list * K + place];
                const double log_sum = s_log[q];
                if (k && isfinite(log_sum))
                    return Choice{ordered((double)s_score[q] + ((double)from_ordered((uint32_t)(k >> 32)) - (double)s_top[q] - log_sum)), q * p.vocab + (int)~(uint32_t)k};
            } else if (s_done[q] && list % SLICES == 0 && place == 0 && isfinite(s_score[q])) {
                return Choice{ordered((double)s_score[q]), q * p.vocab + p.eos};
            }
            return Choice{0ull, 0};
        };
        const int lists = K * SLICES;
        auto logit_of = [&](int list, int place) { return (uint32_t)(s.best[(size_t)list * K + place] >> 32); };
        auto join = [&](auto most) { return join_lists<SLICES, decltype(most)::value>(K, lists, score_of, logit_of, s_chosen, s_chosen_pair); };
        const int n = lists <= 32 ? join(std::integral_constant<int, 1>{}) : lists <= 64 ? join(std::integral_constant<int, 2>{})
                    : lists <= 128 ? join(std::integral_constant<int, 4>{}) : join(std::integral_constant<int, 8>{});
        if (lane == 0) s_found = n;
    }
    __syncthreads();
    const int found = s_found;
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

template <int SLICES, int THREADS, int PT>
amq_status launch_select_as(const SelectParams& p, int batch, int groups, cudaStream_t st)
{
    const size_t smem = select_smem(SLICES, p.beams, nullptr, nullptr);
    auto kernel = beam_select_kernel<SLICES, THREADS, PT>;
    AMQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    AMQ_CUDA_TRY(launch_kernel(kernel, dim3((unsigned)(batch * SLICES)), dim3((unsigned)(THREADS * groups)), smem, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

// MOST: words of a thread and piece
template <int SLICES, int THREADS, int MOST>
amq_status launch_select_groups(const SelectParams& p, int batch, int groups, cudaStream_t st)
{
    if (groups > p.beams) groups = p.beams;
    const int slice = (p.vocab - 1) / SLICES + 1;
    const int pieces = (slice + THREADS * MOST - 1) / (THREADS * MOST), words = ((slice + pieces - 1) / pieces + THREADS - 1) / THREADS;
    if (words <= 2) return launch_select_as<SLICES, THREADS, 2>(p, batch, groups, st);
    if (words <= 5) return launch_select_as<SLICES, THREADS, 5>(p, batch, groups, st);
    if (words <= 8) return launch_select_as<SLICES, THREADS, 8>(p, batch, groups, st);
    if (words <= 10) return launch_select_as<SLICES, THREADS, 10>(p, batch, groups, st);
    if constexpr (MOST > 12) {
        if (words > 21) return launch_select_as<SLICES, THREADS, 24>(p, batch, groups, st);
        if (words > 16) return launch_select_as<SLICES, THREADS, 21>(p, batch, groups, st);
        if (words > 12) return launch_select_as<SLICES, THREADS, 16>(p, batch, groups, st);
    }
    return launch_select_as<SLICES, THREADS, 12>(p, batch, groups, st);
}

amq_status launch_select(const SelectParams& p, int batch, cudaStream_t st)
{
    // Few entries: eight CTAs of all the threads an SM allows, as long as the GPU holds the clusters at once (14 of eight CTAs, 33 of four; a few SMs of every
    // GPC are left over).  Then four CTAs an entry, with as many beams at a time as leave those of all entries on the GPU at once; for many beams, whose lists
    // leave an SM few CTAs, two at least.  By eight and by four CTAs, 8 beams of 9999: 14 entries 9.7 and 10.5 us, 16 13.6 and 10.5; four, two and one
    // beam at a time: 32 entries 11.0, 12.2 and 16.3, 60 20.1, 14.3 and 17.6, 90 27, 22.8 and 19.4; with 16 beams 51, 45.6 and 41.6, of 42000 90, 90 and 105.
    if (batch <= 14) return p.beams > 4 ? launch_select_groups<8, 128, 12>(p, batch, 8, st) : launch_select_groups<8, 256, 12>(p, batch, 4, st);
    return launch_select_groups<4, 256, 24>(p, batch, batch <= 33 ? 4 : batch <= 66 || p.beams > 8 ? 2 : 1, st);
}

// ---- reordering ------------------------------------------------------------------------------------------------------

struct ReorderParams {
    const char* src[AMQ_MAX_STATES]; char* dst[AMQ_MAX_STATES];
    long long src_stride[AMQ_MAX_STATES], dst_stride[AMQ_MAX_STATES];
    int columns[AMQ_MAX_STATES];        // words in a row
    uint32_t wide;                      // states whose rows are words of 16 bytes (a bit each), the others' are of 4
    const int32_t* parents;
    int batch, beams;
};

// A thread owns one column of a batch entry across all its beams: it reads the parents' values first and writes after, so the states may be
// reordered in place without a second copy.  K: registers for the beams.  Bound by memory: four states of 256 x 8 rows of 2048 floats, 67 MB each way, 17 us, 8.0 TB/s
// (what is written is partly still in L2 when the kernel ends); rows of 2047 floats, in words of 4 bytes, 26 to 28 us.
template <typename V, int K>
__device__ __forceinline__ void reorder_columns(const ReorderParams& p)
{
    const int st = blockIdx.y, columns = p.columns[st];
    const long long all = (long long)p.batch * columns;
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < all; at += (long long)gridDim.x * 256) {
        const int entry = (int)(at / columns), column = (int)(at - (long long)entry * columns);
        const long long row0 = (long long)entry * p.beams;
        const char* src = p.src[st] + row0 * p.src_stride[st] + (long long)column * sizeof(V);
        char* dst = p.dst[st] + row0 * p.dst_stride[st] + (long long)column * sizeof(V);
        V v[K];
        int parent[K];
        uint32_t moves = 0;             // beams that are written: all, in place those of another parent
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (b < p.beams) {
                const int q = p.parents[row0 + b];
                parent[b] = q < 0 ? 0 : q < p.beams ? q : p.beams - 1;
            }
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (b < p.beams) {
                v[b] = *reinterpret_cast<const V*>(src + parent[b] * p.src_stride[st]);
                if (parent[b] != b || src != dst) moves |= 1u << b;
            }
#pragma unroll
        for (int b = 0; b < K; ++b)
            if (moves >> b & 1) *reinterpret_cast<V*>(dst + b * p.dst_stride[st]) = v[b];
    }
}

// WIDE, NARROW: whether there are states of either kind (words of 4 bytes alone need fewer registers: 26 us above, 32 with both)
template <int K, bool WIDE, bool NARROW>
__global__ void __launch_bounds__(256)
beam_reorder_kernel(const __grid_constant__ ReorderParams p)
{
    grid_dependency_wait();
    if (WIDE && (!NARROW || (p.wide >> blockIdx.y & 1))) reorder_columns<uint4, K>(p);
    else reorder_columns<uint32_t, K>(p);
}

template <bool WIDE, bool NARROW>
amq_status launch_reorder_as(const ReorderParams& p, int count, cudaStream_t st)
{
    auto kernel = p.beams <= 4 ? beam_reorder_kernel<4, WIDE, NARROW> : p.beams <= 8 ? beam_reorder_kernel<8, WIDE, NARROW>
                : p.beams <= 16 ? beam_reorder_kernel<16, WIDE, NARROW> : beam_reorder_kernel<32, WIDE, NARROW>;
    long long most = 0;
    for (int i = 0; i < count; ++i) if (p.columns[i] > most) most = p.columns[i];
    long long blocks = (most * p.batch + 255) / 256;
    if (blocks > 1 << 20) blocks = 1 << 20;
    AMQ_CUDA_TRY(launch_kernel(kernel, dim3((unsigned)blocks, (unsigned)count), dim3(256), 0, st, true, p));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

amq_status launch_reorder(const ReorderParams& p, int count, cudaStream_t st)
{
    if (p.wide == 0) return launch_reorder_as<false, true>(p, count, st);
    return p.wide == (1u << count) - 1u ? launch_reorder_as<true, false>(p, count, st) : launch_reorder_as<true, true>(p, count, st);
}

}  // namespace
}  // namespace amq

extern "C" {

amq_status amq_beam_select(const float* logits, int ld, int vocab, const float* scores, const int32_t* finished, int eos, int batch, int beams,
                           float* scores_out, int32_t* parents, int32_t* tokens, int32_t* finished_out, void* stream)
{
    if (vocab < 1 || ld < vocab || batch < 0 || beams < 1 || eos < -1 || eos >= vocab || (finished && eos < 0)) return AMQ_ERR_INVALID_ARG;
    if (beams > AMQ_MAX_BEAMS || (long long)beams * vocab > 0x7ffffffell || 8ll * batch > 0x7fffffffll) return AMQ_ERR_UNSUPPORTED;
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
    for (int i = 0; i < count; ++i) {
        if (src_stride[i] < row_bytes[i] || dst_stride[i] < row_bytes[i] || (src[i] == dst[i] && src_stride[i] != dst_stride[i])) return AMQ_ERR_INVALID_ARG;
        if (row_bytes[i] && (!src[i] || !dst[i])) return AMQ_ERR_INVALID_ARG;
        if (row_bytes[i] / 4 > 0x7fffffffu) return AMQ_ERR_UNSUPPORTED;
        const uintptr_t bits = reinterpret_cast<uintptr_t>(src[i]) | reinterpret_cast<uintptr_t>(dst[i]) | row_bytes[i] | src_stride[i] | dst_stride[i];
        if (bits & 3) return AMQ_ERR_ALIGNMENT;
        if ((bits & 15) == 0) p.wide |= 1u << i;
        p.src[i] = static_cast<const char*>(src[i]); p.dst[i] = static_cast<char*>(dst[i]);
        p.src_stride[i] = (long long)src_stride[i]; p.dst_stride[i] = (long long)dst_stride[i];
    }
    // a state that is written twice, or read by another one's threads while its own write it
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j)
            if (i != j && row_bytes[i] && row_bytes[j] && (dst[i] == dst[j] || dst[i] == src[j])) return AMQ_ERR_INVALID_ARG;
    long long most = 0;
    for (int i = 0; i < count; ++i) {
        p.columns[i] = (int)(row_bytes[i] / (p.wide >> i & 1 ? 16 : 4));
        if (p.columns[i] > most) most = p.columns[i];
    }
    if (most == 0) return AMQ_OK;
    return amq::launch_reorder(p, count, (cudaStream_t)stream);
}

}  // extern "C"
