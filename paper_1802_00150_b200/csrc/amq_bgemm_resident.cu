// Batched binary product (Sec. 4, Fig. 3 right; y = sum_i sum_j alpha_i beta_j D_ij + bias) with a resident activation operand
// (amq_resident.cuh).  One CTA per SM; the work is the list of (block of vectors, tile of 128 weight rows) pairs, dealt out in
// equal contiguous shares, so that a CTA expands the activation operand once or twice and streams weight tiles past it.
//
// What bounds it: per tile of 128 rows (32768 x 1024, 512 vectors, 3/2 bits: some 5500 clocks, 3080 of them the tensor pipe's) the chain
// commit - poll - barrier - read - release of every accumulator, and the issue slots that the roles share with the warp that issues the
// MMAs.  That product took 59.8 us with a constant of every operand row added back in the epilogue (twice the instructions, and its
// loads kept the load/store unit busy) and the polling warp on the issuing warp's scheduler; 52.5 us now (behind a flush of L2 65.6 and 59.4).  Outputs leave through shared
// memory as 16-byte pieces.
#include "amq_activation.cuh"
#include "amq_resident.cuh"

namespace amq {

namespace {

struct ResGemmParams {
    ResProblem p;
    const uint32_t* xcodes; const float* xbeta; const float* bias;
    float* y; int ldy;
    int activation; const float* residual; int ldr;     // POST
    int mtiles, blocks;         // tiles of 128 rows, blocks of TB vectors
    int b_bytes;                // expanded activation operand
    int early_weights;          // the kernel before does not write the weights: they may be fetched before it is through
    uint32_t* status;           // set when a bounded wait ran out
};

// Row stride of the results staged for the stores: 8 mod 32 words for two vectors (conflict-free in the m16n8 layout), 16-byte rows.
constexpr int Y_LD = 132;
constexpr int BIAS_BYTES = 2 * 128 * 4;     // POST: bias of a tile's rows, double-buffered
// what lies behind the synchronisation block starts on 16 bytes, as the block does
constexpr int SYNC_BYTES = ((int)sizeof(ResSync) + 15) / 16 * 16;
static_assert(RES_TABLE * 4 % 16 == 0 && RES_ROW_BYTES % 16 == 0 && RES_ALPHA_BYTES % 16 == 0 && Y_LD * 4 % 16 == 0, "");
// groups of eight vectors per epilogue thread: TB <= 64, or 32 (registers)
__host__ __device__ constexpr int res_ng(int k_a) { return k_a <= 2 ? 2 : 1; }

using R = ResRoles<3, 16, 3>;

// VEC: every row of the result (and of the residual) starts on 16 bytes.  (Two kernels, not two paths in one: the registers and instructions of all the roles of a
// kernel of 1024 threads count for each role.  Without VEC a thread stores its four rows one by one; contiguous 128-byte stores, or
// 16-byte pieces shifted against the rows, were slower at most sizes: up to 35 % for rows of 2000 and more.)
template <int KA, bool VEC, bool POST>
__global__ void __launch_bounds__(R::THREADS, 1)
bgemm_resident_kernel(const __grid_constant__ ResGemmParams a)
{
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    const ResProblem& p = a.p;
    constexpr int NG = res_ng(KA);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    float* sBeta = reinterpret_cast<float*>(smem_raw + a.b_bytes);                  // [256] per operand row
    float* sAlpha = sBeta + 256;                                                    // [2][4][128]
    uint32_t* table = reinterpret_cast<uint32_t*>(sAlpha + 2 * AMQ_MAX_K * 128);
    float* sY = reinterpret_cast<float*>(table + RES_TABLE);                        // [TB][Y_LD] results of a tile
    ResSync& sy = *reinterpret_cast<ResSync*>(sY + p.TB * Y_LD);
    float* sBias = reinterpret_cast<float*>(reinterpret_cast<unsigned char*>(&sy) + SYNC_BYTES);    // POST: [2][128]
    float* sR = sBias + 2 * 128;                                                    // POST, where there is a residual: [TB][Y_LD]
    const uint32_t sB = smem_u32(smem_raw);

    // this CTA's share of the (block, tile) list; a pass is the part of it that lies in one block of vectors
    const long long total = (long long)a.blocks * a.mtiles;
    long long w = total * blockIdx.x / gridDim.x;
    const long long w_end = total * (blockIdx.x + 1) / gridDim.x;
    auto pass_tiles = [&](long long at) {
        const int tile0 = (int)(at % a.mtiles);
        return (int)(w_end - at < a.mtiles - tile0 ? w_end - at : a.mtiles - tile0);
    };

    if (tid == 0) res_sync_init<R>(sy);
    res_fill_table(p, table);
    if (warp == R::MMA_WARP) {
        if (!a.early_weights) grid_dependency_wait();       // (a foreign kernel in front may still want tensor memory)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(smem_u32(&sy.tmem_slot)), "r"((uint32_t)RES_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, sy.tmem_slot, 0);
    if (warp < 4) write_unit_scales(tmem, p.ring * p.N, warp);
    __syncthreads();

    // expand the activations of block bb; all threads, ends with a CTA barrier
    auto load_block = [&](int bb) {
        const int b0 = bb * p.TB;
        for (int q = tid; q < p.N; q += R::THREADS) {
            const int b = b0 + res_row_vector<KA>(q), j = res_row_plane<KA>(q);
            sBeta[q] = q < p.TB * KA && b < p.batch ? __ldcg(a.xbeta + (size_t)b * KA + j) : 0.0f;
        }
        res_expand_activations<KA, 1>(p, a.xcodes, (size_t)(p.wpr >> 2), 1, b0, sB);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    // Every role runs its own loop over the passes (the registers of one role are then not held through another's code); a pass
    // ends with a barrier, after which every MMA that read the operand has completed (the epilogue has waited for all
    // accumulators), so the operand may be overwritten.
    bool ok = true;
    if (warp < R::EXP_WARPS) {
        const int r = (warp & 3) * 32 + lane, steps_per_tile = p.k_w * ((p.NS + 1) >> 1);
        int first_step = 0;                         // pipeline steps so far, mod the number of groups
        ResFeedState fs{warp >> 2, 1u};
        ResFeeder<R, RES_PLAIN> feed;
        auto start = [&](long long at) {
            feed.start(p, table, (int)(at % a.mtiles), 1, pass_tiles(at), r, ((warp >> 2) - first_step + R::GROUPS) % R::GROUPS);
        };
        if (!a.early_weights) grid_dependency_wait();
        if (w < w_end) start(w);                    // (no kernel of a chain writes the weights)
        grid_dependency_wait();                     // the planes and coefficients may come from the preceding kernel
        while (w < w_end) {
            load_block((int)(w / a.mtiles));
            ok = res_feed(p, sy, table, feed, tmem, fs);
            const int tiles = pass_tiles(w);
            w += tiles;
            first_step = (int)((first_step + (long long)tiles * steps_per_tile) % R::GROUPS);
            if (w < w_end) start(w);
            if (__syncthreads_or(!ok)) { ok = false; break; }
        }
    } else if (warp == R::MMA_WARP) {
        ResIssueState issue{0, 0, 0, 1};
        grid_dependency_wait();
        while (w < w_end) {
            load_block((int)(w / a.mtiles));
            const int tiles = pass_tiles(w);
            ok = res_issue(p, sy, tiles, tmem, sB, issue);
            w += tiles;
            if (__syncthreads_or(!ok)) { ok = false; break; }
        }
    } else if (warp < R::MMA_WARP) {
        const int te = tid - 32 * R::EXP_WARPS, quarter = warp & 3, sub = (warp - R::EXP_WARPS) >> 2, rl = quarter * 32 + (lane >> 2);
        ResDrainState drain{0, 0};
        uint32_t y_parity = 1;
        // coefficients of a tile's rows: thread te takes one of the 128 k_w, a tile ahead
        auto alpha_of = [&](int tile) {
            const int row = tile * 128 + (te & 127), plane = te >> 7;
            return plane < p.k_w && row < p.units ? __ldcg(p.Walpha + (size_t)row * p.k_w + plane) : 0.0f;
        };
        auto bias_of = [&](int tile) {
            const int row = tile * 128 + te;
            return a.bias && te < 128 && row < p.units ? __ldcg(a.bias + row) : 0.0f;
        };
        grid_dependency_wait();
        while (w < w_end) {
            const int bb = (int)(w / a.mtiles), tile0 = (int)(w % a.mtiles), tiles = pass_tiles(w);
            float next_alpha = alpha_of(tile0), next_bias = POST ? bias_of(tile0) : 0.0f;
            load_block(bb);
            f32x2 beta[NG][KA];
            res_load_beta<R, KA, NG>(p, sBeta, sub, beta);
            for (int t = 0; t < tiles; ++t) {
                float* sa = sAlpha + (t & 1) * AMQ_MAX_K * 128;
                sa[te] = next_alpha;
                if (POST && te < 128) sBias[(t & 1) * 128 + te] = next_bias;
                if (res_epi_bar<R>(!ok)) { ok = false; break; }        // (also: everybody is past the tile before last, whose buffer this is)
                if (t + 1 < tiles) { next_alpha = alpha_of(tile0 + t + 1); if (POST) next_bias = bias_of(tile0 + t + 1); }
                f32x2 y[NG][4];
                ok = res_drain_tile<R, KA, NG>(p, sy, sa, quarter, sub, tmem, beta, drain, y);
                if constexpr (POST) {
                    if (ok) {
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            float v[8];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float bias = sBias[(t & 1) * 128 + rl + 8 * i];       // added here, in front of the activation
                                unpack2(y[g][i], v[2 * i], v[2 * i + 1]);
                                v[2 * i] += bias; v[2 * i + 1] += bias;
                            }
                            activate(v, a.activation);
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[g][i] = pack2(v[2 * i], v[2 * i + 1]);
                        }
                    }
                }
                // Results leave through shared memory and three warps of their own: in this layout a store from the registers is four
                // 32-byte pieces, and stores from the epilogue warps held them up for longer than a tile's MMAs take.
                if (ok && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&sy.yempty), y_parity))) { *(volatile int*)&sy.failed = 1; ok = false; }
                y_parity ^= 1u;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const int e = (R::SPLIT * g + sub) * 8 + 2 * (lane & 3);
                    if (e >= p.TB) break;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float y0, y1;
                        unpack2(y[g][i], y0, y1);
                        sY[e * Y_LD + rl + 8 * i] = y0;
                        sY[(e + 1) * Y_LD + rl + 8 * i] = y1;
                    }
                }
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(&sy.yfull)) : "memory");
            }
            w += tiles;
            if (__syncthreads_or(!ok)) { ok = false; break; }
        }
    } else {
        uint32_t y_parity = 0;
        while (w < w_end) {
            const int bb = (int)(w / a.mtiles), tile0 = (int)(w % a.mtiles), b0 = bb * p.TB, tiles = pass_tiles(w);
            grid_dependency_wait();
            load_block(bb);
            const int last = p.batch - b0 < p.TB ? p.batch - b0 : p.TB;
            auto store = [&](int e, int row, bool vec, const float4& v) {
                float* out = a.y + (size_t)(b0 + e) * a.ldy + row;
                if (vec) {
                    *reinterpret_cast<float4*>(out) = v;
                } else {
                    if (row < p.units) out[0] = v.x;
                    if (row + 1 < p.units) out[1] = v.y;
                    if (row + 2 < p.units) out[2] = v.z;
                    if (row + 3 < p.units) out[3] = v.w;
                }
            };
            // The residual of a tile comes by asynchronous copies, a tile ahead, each lane's to where that lane will read it: a window of loads in registers left
            // these three warps waiting (32768 x 1024, 512 vectors, residual alone: 85 us, 71 so).  It may be y itself: every element is read by the thread that
            // writes it, before.
            const int first = warp - R::MMA_WARP - 1;
            auto fetch = [&](int t, int e) {
                const int row = (tile0 + t) * 128 + 4 * lane;
                const uint32_t to = smem_u32(sR + e * Y_LD + 4 * lane);
                const float* from = a.residual + (size_t)(b0 + e) * a.ldr + row;
                if (VEC && row + 3 < p.units) {
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
                } else {
                    for (int q = 0; q < 4 && row + q < p.units; ++q)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(to + 4 * q), "l"(from + q) : "memory");
                }
            };
            if (POST && a.residual)
                for (int e = first; e < last; e += R::OUT_WARPS) fetch(0, e);
            for (int t = 0; t < tiles && ok; ++t) {
                const int row = (tile0 + t) * 128 + 4 * lane;
                const bool vec = VEC && row + 3 < p.units;
                if constexpr (POST) {
                    ok = __all_sync(0xffffffffu, mbar_wait_relaxed(smem_u32(&sy.yfull), y_parity, &sy.failed));
                    y_parity ^= 1u;
                    asm volatile("cp.async.wait_all;" ::: "memory");        // (a wait that ran out leaves no copies in flight either)
                    if (!ok) { *(volatile int*)&sy.failed = 1; break; }
#pragma unroll 4
                    for (int e = first; e < last; e += R::OUT_WARPS) {
                        float4 v = *reinterpret_cast<const float4*>(sY + e * Y_LD + 4 * lane);
                        if (a.residual) {
                            const float4 r = *reinterpret_cast<const float4*>(sR + e * Y_LD + 4 * lane);
                            v.x += r.x; v.y += r.y; v.z += r.z; v.w += r.w;
                            if (t + 1 < tiles) fetch(t + 1, e);
                        }
                        store(e, row, vec, v);
                    }
                    __syncwarp();
                    if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(&sy.yempty)) : "memory");
                    continue;
                }
                float4 bias = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (a.bias) {
                    if (row < p.units) bias.x = __ldcg(a.bias + row);
                    if (row + 1 < p.units) bias.y = __ldcg(a.bias + row + 1);
                    if (row + 2 < p.units) bias.z = __ldcg(a.bias + row + 2);
                    if (row + 3 < p.units) bias.w = __ldcg(a.bias + row + 3);
                }
                ok = __all_sync(0xffffffffu, mbar_wait_relaxed(smem_u32(&sy.yfull), y_parity, &sy.failed));
                y_parity ^= 1u;
                if (!ok) { *(volatile int*)&sy.failed = 1; break; }
#pragma unroll 4
                for (int e = warp - R::MMA_WARP - 1; e < last; e += R::OUT_WARPS) {
                    float4 v = *reinterpret_cast<const float4*>(sY + e * Y_LD + 4 * lane);
                    v.x += bias.x; v.y += bias.y; v.z += bias.z; v.w += bias.w;
                    store(e, row, vec, v);
                }
                __syncwarp();
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(&sy.yempty)) : "memory");
            }
            w += tiles;
            if (__syncthreads_or(!ok)) { ok = false; break; }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (!ok) {      // (uniform) give the tensor core time to drain before tensor memory is released
        if (tid == 0) atomicExch(a.status, 1u);
        __nanosleep(1000000);
        __syncthreads();
    }
    if (warp == R::MMA_WARP)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"((uint32_t)RES_TMEM_COLS) : "memory");
}

struct ResGemmPlan { ResGemmParams a; int grid; size_t smem; bool vec_out; };

bool plan(const GemmArgs& g, int sms, ResGemmPlan* out)
{
    if (g.epilogue != EPI_Y) return false;
    ResGemmParams a{};
    ResProblem& p = a.p;
    p.W = g.Wcodes; p.Walpha = g.Walpha; p.k_w = g.k_w; p.wpr = words_per_row(g.n);
    p.vec32 = p.wpr % 8 == 0 && (reinterpret_cast<uintptr_t>(g.Wcodes) & 31) == 0;
    p.cell = RES_PLAIN; p.units = g.m;
    p.n = g.n; p.NS = (g.n + 255) / 256; p.batch = g.batch;
    a.mtiles = (g.m + 127) / 128;
    auto post_bytes = [&](int TB) { return (size_t)TB * Y_LD * 4 * (g.post && g.residual ? 2 : 1) + (g.post ? BIAS_BYTES + 16 : 0); };
    // block of vectors: the size with the least estimated time (shares of tiles x steps, plus the expansion of the operand,
    // which a share pays at least once); sizes whose operand does not fit shared memory are out (n > 28000 or so: none fits)
    double best = 0.0;
    for (int TB = 8; TB <= 8 * res_ng(g.k_a) * R::SPLIT; TB += 8) {
        ResProblem q = p;
        if (!res_set_block<R>(q, TB, g.k_a, post_bytes(TB))) break;
        const long long blocks = (g.batch + TB - 1) / TB, per_cta = (blocks * a.mtiles + sms - 1) / sms;
        const double expand = (double)q.N * q.NS * 128 / 80.0 + 1500.0;
        const double t = (double)per_cta * q.k_w * q.NS * res_slot_clocks(q) + expand * (1.0 + (double)per_cta / a.mtiles);
        if (best == 0.0 || t < best) { best = t; a.p = q; a.blocks = (int)blocks; }
        if (TB >= g.batch) break;
    }
    if (best == 0.0) return false;
    a.b_bytes = a.p.NS * a.p.N * 128;
    a.xcodes = g.xcodes; a.xbeta = g.xbeta; a.bias = g.bias; a.y = g.y; a.ldy = g.ldy;
    const long long total = (long long)a.blocks * a.mtiles;
    out->grid = (int)(total < sms ? total : sms);
    out->smem = res_smem_bytes(a.p) + post_bytes(a.p.TB);
    a.early_weights = !g.from_entry;
    a.activation = g.activation; a.residual = g.residual; a.ldr = g.ldr;
    out->vec_out = aligned16(g.y) && g.ldy % 4 == 0 && (!g.residual || (aligned16(g.residual) && g.ldr % 4 == 0));
    out->a = a;
    return true;
}

template <int KA, bool POST>
amq_status launch(const ResGemmPlan& pl, bool overlap, cudaStream_t st)
{
    auto kernel = pl.vec_out ? bgemm_resident_kernel<KA, true, POST> : bgemm_resident_kernel<KA, false, POST>;
    AMQ_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pl.smem));
    AMQ_CUDA_TRY(launch_kernel(kernel, dim3((unsigned)pl.grid), dim3(R::THREADS), pl.smem, st, overlap, pl.a));
    AMQ_LAUNCH_CHECK();
    return AMQ_OK;
}

}  // namespace

double gemm_resident_clocks(const GemmArgs& g, int sms)
{
    // from 16 vectors on always; for 2..15 vectors when the weight matrix is large enough that the CUDA-core kernel's tile loop
    // costs more than this kernel's set-up
    if (sms < 1) sms = res_sm_count();
    ResGemmPlan pl;
    const bool big = (long long)g.m * g.k_w * words_per_row(g.n) >= (1ll << 17);
    if (!(g.batch >= 16 || (g.batch >= 2 && big)) || !plan(g, sms, &pl)) return 0.0;
    const ResProblem& p = pl.a.p;
    const double tiles = (double)(((long long)pl.a.blocks * pl.a.mtiles + sms - 1) / sms), passes = 1.0 + (tiles - 1.0) / pl.a.mtiles;
    return passes * (15600.0 + 7.4 * p.N * p.NS) + 23.8 * p.k_w * p.NS +
           tiles * (p.k_w * (1.11 * p.NS * res_slot_clocks(p) + 0.3 * p.N + 607.0) + 31.0 * p.TB);
}

amq_status launch_binary_gemm_resident(const GemmArgs& g, cudaStream_t st)
{
    ResGemmPlan pl;
    if (!plan(g, res_sm_count(), &pl)) return AMQ_ERR_UNSUPPORTED;
    amq_status s = tc_status_word(&pl.a.status);
    if (s != AMQ_OK) return s;
    const bool overlap = g.overlap_with_previous || g.from_entry;
    switch (g.k_a) {
        case 1: return g.post ? launch<1, true>(pl, overlap, st) : launch<1, false>(pl, overlap, st);
        case 2: return g.post ? launch<2, true>(pl, overlap, st) : launch<2, false>(pl, overlap, st);
        case 3: return g.post ? launch<3, true>(pl, overlap, st) : launch<3, false>(pl, overlap, st);
        case 4: return g.post ? launch<4, true>(pl, overlap, st) : launch<4, false>(pl, overlap, st);
    }
    return AMQ_ERR_UNSUPPORTED;
}

}  // namespace amq
