// Group normalisation with an activation, channels last, and its gradients.
#include "elem.cuh"

namespace {

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    float *mean, *rstd;
    float *part;  // gradients of gamma and beta of each image, [2][B][C]
    long long ldx, ldy;
    int B, HW, C, groups, per, act;
    float eps;
};

constexpr int kNormThreads = 256;

// Sum over the block, the same in every thread; tmp holds one value per warp.
__device__ __forceinline__ float block_sum(float v, float *tmp) {
    v = warp_sum(v);
    __syncthreads();
    if (threadIdx.x % 32 == 0) tmp[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < kNormThreads / 32; ++i) v += tmp[i];
    return v;
}

__device__ __forceinline__ float activate(float z, int act) {
    return act == PPO_ACT_RELU ? fmaxf(z, 0.f) : act == PPO_ACT_SILU ? z / (1.f + expf(-z)) : z;
}

// Which side of 0 gamma xhat + beta is on: rounding to 32 bits decides it wrongly only within a few units of the last place of its
// terms, and there 64 bits do.
__device__ __forceinline__ bool relu_open(float x, float mean, float rstd, float gamma, float beta, float z) {
    if (fabsf(z) > 1e-6f * (fabsf(gamma) * rstd * (fabsf(x) + fabsf(mean)) + fabsf(beta))) return z > 0.f;
    return ((double)x - (double)mean) * (double)rstd * (double)gamma + (double)beta > 0.;
}

template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_kernel(NormArgs a) {
    grid_wait();
    __shared__ float tmp[kNormThreads / 32];
    const int b = blockIdx.x / a.groups, g = blockIdx.x % a.groups, c0 = g * a.per;
    const T *x = static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0;
    T *y = static_cast<T *>(a.y) + (long long)b * a.HW * a.ldy + c0;
    const long long n = (long long)a.HW * a.per;
    float s = 0.f;
    for (long long i = threadIdx.x; i < n; i += kNormThreads) s += to_f32(x[i / a.per * a.ldx + i % a.per]);
    const float mean = block_sum(s, tmp) / (float)n;
    s = 0.f;
    for (long long i = threadIdx.x; i < n; i += kNormThreads) {
        const float d = to_f32(x[i / a.per * a.ldx + i % a.per]) - mean;
        s += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum(s, tmp) / (float)n + a.eps);
    if (threadIdx.x == 0) {
        a.mean[blockIdx.x] = mean;
        a.rstd[blockIdx.x] = rstd;
    }
    for (long long i = threadIdx.x; i < n; i += kNormThreads) {
        const int c = (int)(i % a.per);
        const float xhat = (to_f32(x[i / a.per * a.ldx + c]) - mean) * rstd;
        const float z = a.gamma ? xhat * a.gamma[c0 + c] + a.beta[c0 + c] : xhat;
        y[i / a.per * a.ldy + c] = from_f32<T>(activate(z, a.act));
    }
}

template <typename T>
struct Grad {
    const T *x, *dy;
    float mean, rstd;
    int act;
    // xhat and dL/dz of one element
    __device__ __forceinline__ void at(long long ix, long long iy, float gamma, float beta, float &xhat, float &dz) const {
        const float v = to_f32(x[ix]);
        xhat = (v - mean) * rstd;
        const float z = gamma * xhat + beta;
        dz = to_f32(dy[iy]);
        if (act == PPO_ACT_RELU) {
            if (!relu_open(v, mean, rstd, gamma, beta, z)) dz = 0.f;
        } else if (act == PPO_ACT_SILU) {
            const float p = 1.f / (1.f + expf(-z));
            dz *= p * (1.f + z * (1.f - p));
        }
    }
};

template <typename T>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_kernel(NormArgs a) {
    grid_wait();
    __shared__ float tmp[kNormThreads / 32];
    const int b = blockIdx.x / a.groups, g = blockIdx.x % a.groups, c0 = g * a.per;
    const Grad<T> f = {static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0, static_cast<const T *>(a.dy) + (long long)b * a.HW * a.ldy + c0,
                       a.mean[blockIdx.x], a.rstd[blockIdx.x], a.act};
    T *dx = static_cast<T *>(a.dx) + (long long)b * a.HW * a.ldx + c0;
    float m1 = 0.f, m2 = 0.f;
    for (int c = 0; c < a.per; ++c) {
        const float gamma = a.gamma ? a.gamma[c0 + c] : 1.f, beta = a.gamma ? a.beta[c0 + c] : 0.f;
        float s1 = 0.f, s2 = 0.f;
        for (int i = threadIdx.x; i < a.HW; i += kNormThreads) {
            float xhat, dz;
            f.at(i * a.ldx + c, i * a.ldy + c, gamma, beta, xhat, dz);
            s1 += dz;
            s2 += dz * xhat;
        }
        s1 = block_sum(s1, tmp);
        s2 = block_sum(s2, tmp);
        if (a.part && threadIdx.x == 0) {
            a.part[(size_t)b * a.C + c0 + c] = s2;
            a.part[((size_t)a.B + b) * a.C + c0 + c] = s1;
        }
        m1 += gamma * s1;
        m2 += gamma * s2;
    }
    const long long n = (long long)a.HW * a.per;
    m1 /= (float)n;
    m2 /= (float)n;
    __syncthreads();  // dx may be dy
    for (long long i = threadIdx.x; i < n; i += kNormThreads) {
        const int c = (int)(i % a.per);
        const float gamma = a.gamma ? a.gamma[c0 + c] : 1.f, beta = a.gamma ? a.beta[c0 + c] : 0.f;
        float xhat, dz;
        f.at(i / a.per * a.ldx + c, i / a.per * a.ldy + c, gamma, beta, xhat, dz);
        dx[i / a.per * a.ldx + c] = from_f32<T>(f.rstd * (gamma * dz - m1 - xhat * m2));
    }
}

// Sums over the images, a thread per channel.
__global__ void __launch_bounds__(128) norm_sum_kernel(const float *part, int B, int C, float *dgamma, float *dbeta, int accumulate) {
    grid_wait();
    const int c = blockIdx.x * 128 + threadIdx.x;
    if (c >= C) return;
    for (int k = 0; k < 2; ++k) {
        double s = 0;
        for (int b = 0; b < B; ++b) s += part[((size_t)k * B + b) * C + c];
        float *out = k == 0 ? dgamma : dbeta;
        out[c] = (float)(s + (accumulate ? (double)out[c] : 0.));
    }
}

int check(const ppo_group_norm_desc *d) {
    if (!d || d->B <= 0 || d->HW <= 0 || d->C <= 0 || d->groups <= 0) return PPO_ERR_INVALID_ARG;
    if (d->act < PPO_ACT_NONE || d->act > PPO_ACT_SILU || d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->C % d->groups != 0 || d->ldx < d->C || d->ldy < d->C) return PPO_ERR_SHAPE;
    if ((long long)d->B * d->groups > 0x7fffffffll) return PPO_ERR_UNSUPPORTED;
    return PPO_OK;
}

NormArgs args(const ppo_group_norm_desc *d) {
    NormArgs a = {};
    a.ldx = d->ldx;
    a.ldy = d->ldy;
    a.B = d->B;
    a.HW = d->HW;
    a.C = d->C;
    a.groups = d->groups;
    a.per = d->C / d->groups;
    a.act = d->act;
    return a;
}

}  // namespace

extern "C" size_t ppo_group_norm_workspace_bytes(const ppo_group_norm_desc *d, int backward) {
    if (check(d) != PPO_OK || !backward) return 0;
    return (size_t)2 * d->B * d->C * sizeof(float);
}

extern "C" int ppo_group_norm_fwd(const ppo_group_norm_desc *d, float eps, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                                  float *rstd, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    if (!x || !y || !mean || !rstd || !gamma != !beta || !(eps >= 0.f)) return PPO_ERR_INVALID_ARG;
    if (x == y && d->ldx != d->ldy) return PPO_ERR_SHAPE;
    const size_t need = ppo_group_norm_workspace_bytes(d, 0), e = elem_bytes(d->dtype);
    if (need > 0 && !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd})
        if (!ppo_aligned(p, 4)) return PPO_ERR_ALIGN;
    if (!ppo_aligned(x, e) || !ppo_aligned(y, e) || !ppo_aligned(workspace, 16)) return PPO_ERR_ALIGN;
    NormArgs a = args(d);
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = eps;
    return with_elem(d->dtype, [&](auto t) {
        return ppo_launch(norm_fwd_kernel<decltype(t)>, dim3(d->B * d->groups), dim3(kNormThreads), 0, static_cast<cudaStream_t>(stream), a);
    });
}

extern "C" int ppo_group_norm_bwd(const ppo_group_norm_desc *d, const void *x, const float *gamma, const float *beta, const float *mean,
                                  const float *rstd, const void *dy, void *dx, float *dgamma, float *dbeta, int accumulate, void *workspace,
                                  size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    if (!x || !mean || !rstd || !dy || !dx || !gamma != !beta || !dgamma != !dbeta) return PPO_ERR_INVALID_ARG;
    if (dx == dy && d->ldx != d->ldy) return PPO_ERR_SHAPE;
    const size_t need = ppo_group_norm_workspace_bytes(d, 1), e = elem_bytes(d->dtype);
    if (need > 0 && !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd, (const void *)dgamma, (const void *)dbeta})
        if (!ppo_aligned(p, 4)) return PPO_ERR_ALIGN;
    if (!ppo_aligned(x, e) || !ppo_aligned(dy, e) || !ppo_aligned(dx, e) || !ppo_aligned(workspace, 16)) return PPO_ERR_ALIGN;
    NormArgs a = args(d);
    a.x = x;
    a.dy = dy;
    a.dx = dx;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.part = dgamma ? static_cast<float *>(workspace) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    PPO_TRY(with_elem(d->dtype, [&](auto t) {
        return ppo_launch(norm_bwd_kernel<decltype(t)>, dim3(d->B * d->groups), dim3(kNormThreads), 0, st, a);
    }));
    if (!dgamma) return PPO_OK;
    return ppo_launch(norm_sum_kernel, dim3(ppo_cdiv(d->C, 128)), dim3(128), 0, st, (const float *)a.part, (int)d->B, (int)d->C, dgamma, dbeta,
                      accumulate);
}
