#include "param_sum.cuh"

namespace {

// 32 columns a block, every so many shares a warp.
template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) param_sum_kernel(const float *part, int parts, ParamSums s, int accumulate) {
    grid_wait();
    __shared__ double sum[WARPS][32];
    const long long n = s.n[0] + s.n[1] + s.n[2];
    const int l = threadIdx.x % 32, w = threadIdx.x / 32;
    long long i = (long long)blockIdx.x * 32 + l;
    double v = 0;
    if (i < n) {
#pragma unroll 8
        for (int p = w; p < parts; p += WARPS) v += part[p * n + i];
    }
    sum[w][l] = v;
    __syncthreads();
    if (w > 0 || i >= n) return;
    for (int k = 1; k < WARPS; ++k) v += sum[k][l];
    int k = 0;
    for (; k < 2 && i >= s.n[k]; ++k) i -= s.n[k];
    float *out = k == 0 ? s.out[0] : k == 1 ? s.out[1] : s.out[2];
    if (out) out[i] = (float)(v + (accumulate ? (double)out[i] : 0.));
}

}  // namespace

int ppo_param_sum(const float *part, int parts, const ParamSums &s, int accumulate, cudaStream_t st) {
    const long long n = s.n[0] + s.n[1] + s.n[2];
    const dim3 grid((unsigned)((n + 31) / 32));
    // 296 shares of 128 columns: 10.0 us by eight warps, 5.2 by 32; 37 shares of 10240: 5.4 and 5.8
    if (parts > 64) return ppo_launch(param_sum_kernel<32>, grid, dim3(1024), 0, st, part, parts, s, accumulate);
    return ppo_launch(param_sum_kernel<8>, grid, dim3(256), 0, st, part, parts, s, accumulate);
}
