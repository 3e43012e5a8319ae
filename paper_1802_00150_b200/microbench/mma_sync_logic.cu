// Microbenchmark: the integer mma.sync of the cache attention (m16n8k32, s8 by u8) alone and beside the instructions that make its operands: SM clocks per MMA,
// four independent chains a warp, 4 to 16 warps an SM, one CTA on every SM.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cuda_runtime.h>
#define CK(x) do { cudaError_t e_ = (x); if (e_ != cudaSuccess) { printf("CUDA error %s at %d\n", cudaGetErrorString(e_), __LINE__); exit(1); } } while (0)
constexpr int ITERS = 512, CHAINS = 4, SMS = 148, MAX_WARPS = 16;

// ANDS logic instructions and FMAS fp32 ones for every MMA; MMA = false: those alone
template <bool MMA, int ANDS, int FMAS>
__global__ void __launch_bounds__(32 * MAX_WARPS) k(int* out, long long* clk, uint32_t seed)
{
    const uint32_t a[4] = {seed, seed + 1, seed + 2, seed + 3};
    int d[CHAINS][4];
    uint32_t w[8];
    float f[8];
    for (int c = 0; c < CHAINS; ++c) for (int i = 0; i < 4; ++i) d[c][i] = c + i;
    for (int i = 0; i < 8; ++i) { w[i] = seed * (i + 1) + threadIdx.x; f[i] = (float)w[i]; }
    __syncthreads();
    const long long t0 = clock64();
#pragma unroll 1
    for (int it = 0; it < ITERS; ++it) {
#pragma unroll
        for (int c = 0; c < CHAINS; ++c) {
            if (MMA)
                asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                             : "+r"(d[c][0]), "+r"(d[c][1]), "+r"(d[c][2]), "+r"(d[c][3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(w[c]), "r"(w[c + 1]));
#pragma unroll
            for (int i = 0; i < ANDS; ++i) asm volatile("lop3.b32 %0, %0, %1, %2, 0x96;" : "+r"(w[(c + i) & 7]) : "r"(a[i & 3]), "r"(seed));
#pragma unroll
            for (int i = 0; i < FMAS; ++i) asm volatile("fma.rn.f32 %0, %0, %1, %2;" : "+f"(f[(c + i) & 7]) : "f"(1.0001f), "f"(0.5f));
        }
    }
    __syncthreads();
    const long long t1 = clock64();
    int s = 0;
    for (int c = 0; c < CHAINS; ++c) for (int i = 0; i < 4; ++i) s += d[c][i];
    for (int i = 0; i < 8; ++i) s += (int)w[i] + (int)f[i];
    out[blockIdx.x * blockDim.x + threadIdx.x] = s;
    if (threadIdx.x == 0) clk[blockIdx.x] = t1 - t0;
}

template <bool MMA, int ANDS, int FMAS> void run(int warps)
{
    int* out;
    long long *clk, h[SMS];
    CK(cudaMalloc(&out, sizeof(int) * SMS * 32 * MAX_WARPS));
    CK(cudaMalloc(&clk, sizeof(h)));
    for (int i = 0; i < 2; ++i) k<MMA, ANDS, FMAS><<<SMS, warps * 32>>>(out, clk, 12345);
    CK(cudaGetLastError());
    CK(cudaDeviceSynchronize());
    CK(cudaMemcpy(h, clk, sizeof(h), cudaMemcpyDeviceToHost));
    printf("%s, %d logic, %d fma beside it, %2d warps: %.2f clocks of an SM each\n", MMA ? "MMA" : "no MMA", ANDS, FMAS, warps, (double)h[0] / ((double)ITERS * CHAINS * warps));
    CK(cudaFree(out));
    CK(cudaFree(clk));
}

int main()
{
    for (int warps : {4, 8, 16}) run<true, 0, 0>(warps);
    run<true, 2, 0>(16); run<true, 4, 0>(16); run<true, 0, 4>(16); run<true, 2, 4>(16);
    run<false, 2, 0>(16); run<false, 4, 0>(16); run<false, 0, 4>(16); run<false, 2, 4>(16);
    return 0;
}
