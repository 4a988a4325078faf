// Norms of queries and keys for each head with the rotation by their positions, and the gradients.
//
// Angles in 64 bits down to the fraction of a turn, which fits 32; the rest in 32 bits; what is stored is rounded once.
#include "elem.cuh"
#include "param_sum.cuh"

namespace {

constexpr int kMaxD = 256;

struct QkArgs {
    const void *q, *k, *dqo, *dko;
    void *qo, *ko, *dq, *dk;
    const float *gamma_q, *gamma_k;
    const int32_t *pos;
    const double *freq;
    float *part;  // shares of the gradients of gamma, [blocks][2][d]
    long long ldq, ldk, ldqo, ldko;
    int rows, heads, kv, d, pairs, interleaved;
    float eps;
};

// cos and sin of pos * freq.
__device__ __forceinline__ float2 turn(int pos, double freq) {
    const double t = (double)pos * freq * 0.15915494309189535;  // turns
    float2 r;
    sincospif((float)(2. * (t - rint(t))), &r.y, &r.x);
    return r;
}

// Where element i of a head stands in the rotation: its pair, and which of the two it is; pair -1: it stays.
struct Place {
    int pair, other;
    bool second;
};
__device__ __forceinline__ Place place(const QkArgs &a, int i) {
    if (i >= 2 * a.pairs) return {-1, i, false};
    if (a.interleaved) return {i / 2, i ^ 1, (i & 1) != 0};
    return i < a.pairs ? Place{i, i + a.pairs, false} : Place{i - a.pairs, i - a.pairs, true};
}

// ---- any size and alignment: a warp per head, element by element ----

template <typename T>
__global__ void __launch_bounds__(256) qk_fwd_any_kernel(QkArgs a) {
    grid_wait();
    __shared__ float all[8][kMaxD];
    const int lane = threadIdx.x % 32, per = a.heads + a.kv;
    float *n = all[threadIdx.x / 32];
    const long long items = (long long)a.rows * per;
    for (long long item = (long long)blockIdx.x * 8 + threadIdx.x / 32; item < items; item += (long long)gridDim.x * 8) {
        const long long row = item / per;
        const int h = (int)(item - row * per);
        const bool key = h >= a.heads;
        const T *x = key ? static_cast<const T *>(a.k) + row * a.ldk + (h - a.heads) * a.d : static_cast<const T *>(a.q) + row * a.ldq + h * a.d;
        T *y = key ? static_cast<T *>(a.ko) + row * a.ldko + (h - a.heads) * a.d : static_cast<T *>(a.qo) + row * a.ldqo + h * a.d;
        const float *gamma = key ? a.gamma_k : a.gamma_q;
        float s = 0.f;
        for (int i = lane; i < a.d; i += 32) {
            n[i] = to_f32(x[i]);
            s = fmaf(n[i], n[i], s);
        }
        const float r = 1.f / sqrtf(warp_sum(s) / (float)a.d + a.eps);
        for (int i = lane; i < a.d; i += 32) n[i] *= r * (gamma ? gamma[i] : 1.f);
        __syncwarp();
        for (int i = lane; i < a.d; i += 32) {
            const Place p = place(a, i);
            float v = n[i];
            if (p.pair >= 0) {
                const float2 t = turn(a.pos[row], a.freq[p.pair]);
                v = p.second ? fmaf(n[p.other], t.y, v * t.x) : fmaf(-n[p.other], t.y, v * t.x);
            }
            y[i] = from_f32<T>(v);
        }
        __syncwarp();
    }
}

template <typename T>
__global__ void __launch_bounds__(256) qk_bwd_any_kernel(QkArgs a) {
    grid_wait();
    __shared__ float all[8][kMaxD];
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32, per = a.heads + a.kv;
    float *n = all[w], sum[2][kMaxD / 32] = {};
    const long long items = (long long)a.rows * per;
    for (long long item = (long long)blockIdx.x * 8 + w; item < items; item += (long long)gridDim.x * 8) {
        const long long row = item / per;
        const int h = (int)(item - row * per);
        const bool key = h >= a.heads;
        const T *x = key ? static_cast<const T *>(a.k) + row * a.ldk + (h - a.heads) * a.d : static_cast<const T *>(a.q) + row * a.ldq + h * a.d;
        const T *dy = key ? static_cast<const T *>(a.dko) + row * a.ldko + (h - a.heads) * a.d : static_cast<const T *>(a.dqo) + row * a.ldqo + h * a.d;
        T *dx = key ? static_cast<T *>(a.dk) + row * a.ldk + (h - a.heads) * a.d : static_cast<T *>(a.dq) + row * a.ldq + h * a.d;
        const float *gamma = key ? a.gamma_k : a.gamma_q;
        float v[kMaxD / 32], s = 0.f;
#pragma unroll
        for (int j = 0; j < kMaxD / 32; ++j) {
            const int i = lane + 32 * j;
            v[j] = i < a.d ? to_f32(x[i]) : 0.f;
            if (i < a.d) n[i] = to_f32(dy[i]);
            s = fmaf(v[j], v[j], s);
        }
        const float r = 1.f / sqrtf(warp_sum(s) / (float)a.d + a.eps);
        __syncwarp();
        float g[kMaxD / 32], dot = 0.f;
#pragma unroll
        for (int j = 0; j < kMaxD / 32; ++j) {
            const int i = lane + 32 * j;
            g[j] = 0.f;
            if (i >= a.d) continue;
            const Place p = place(a, i);
            g[j] = n[i];
            if (p.pair >= 0) {
                const float2 t = turn(a.pos[row], a.freq[p.pair]);
                g[j] = p.second ? fmaf(-n[p.other], t.y, g[j] * t.x) : fmaf(n[p.other], t.y, g[j] * t.x);
            }
            v[j] *= r;
            sum[key][j] = fmaf(g[j], v[j], sum[key][j]);
            g[j] *= gamma ? gamma[i] : 1.f;
            dot = fmaf(g[j], v[j], dot);
        }
        dot = warp_sum(dot) / (float)a.d;
#pragma unroll
        for (int j = 0; j < kMaxD / 32; ++j) {
            const int i = lane + 32 * j;
            if (i < a.d) dx[i] = from_f32<T>(r * fmaf(-v[j], dot, g[j]));
        }
        __syncwarp();
    }
    if (!a.part) return;
    for (int key = 0; key < 2; ++key) {
        __syncthreads();
        for (int j = 0; j < kMaxD / 32; ++j)
            if (lane + 32 * j < a.d) n[lane + 32 * j] = sum[key][j];
        __syncthreads();
        for (int i = threadIdx.x; i < a.d; i += 256) {
            float s = 0.f;
            for (int k = 0; k < 8; ++k) s += all[k][i];
            a.part[((size_t)blockIdx.x * 2 + key) * a.d + i] = s;
        }
    }
}

int check(const ppo_qk_norm_desc *d) {
    if (!d || d->rows <= 0 || d->heads <= 0 || d->kv_heads <= 0 || d->d <= 0 || d->pairs < 0) return PPO_ERR_INVALID_ARG;
    if (d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->d > kMaxD || d->heads > 0xffffff || d->kv_heads > 0xffffff) return PPO_ERR_UNSUPPORTED;
    const int64_t wq = (int64_t)d->heads * d->d, wk = (int64_t)d->kv_heads * d->d;
    if (2 * (int64_t)d->pairs > d->d || d->ldq < wq || d->ldqo < wq || d->ldk < wk || d->ldko < wk) return PPO_ERR_SHAPE;
    return PPO_OK;
}
bool misaligned(std::initializer_list<const void *> ps, size_t a) {
    for (const void *p : ps)
        if (!ppo_aligned(p, a)) return true;
    return false;
}

QkArgs args(const ppo_qk_norm_desc *d, float eps, const void *q, const void *k, const float *gamma_q, const float *gamma_k, const int32_t *pos,
            const double *freq) {
    QkArgs a = {};
    a.q = q;
    a.k = k;
    a.gamma_q = gamma_q;
    a.gamma_k = gamma_k;
    a.pos = pos;
    a.freq = freq;
    a.ldq = d->ldq;
    a.ldk = d->ldk;
    a.ldqo = d->ldqo;
    a.ldko = d->ldko;
    a.rows = d->rows;
    a.heads = d->heads;
    a.kv = d->kv_heads;
    a.d = d->d;
    a.pairs = d->pairs;
    a.interleaved = d->interleaved;
    a.eps = eps;
    return a;
}

// Blocks of a call with gradients of gamma: by sizes alone, so that the order of the sums goes by them.
int blocks_of(const ppo_qk_norm_desc *d) {
    const long long all = ((long long)d->rows * (d->heads + d->kv_heads) + 7) / 8;
    return (int)(all < 4 * 148 ? all : 4 * 148);
}

}  // namespace

extern "C" size_t ppo_qk_norm_rotate_workspace_bytes(const ppo_qk_norm_desc *d) {
    return check(d) == PPO_OK ? (size_t)blocks_of(d) * 2 * d->d * sizeof(float) : 0;
}

extern "C" int ppo_qk_norm_rotate_fwd(const ppo_qk_norm_desc *d, float eps, const void *q, const void *k, const float *gamma_q, const float *gamma_k,
                                      const int32_t *pos, const double *freq, void *q_out, void *k_out, void *stream) {
    PPO_TRY(check(d));
    if (!q || !k || !q_out || !k_out || (d->pairs > 0 && (!pos || !freq)) || !(eps >= 0.f)) return PPO_ERR_INVALID_ARG;
    if ((q == q_out && d->ldq != d->ldqo) || (k == k_out && d->ldk != d->ldko)) return PPO_ERR_SHAPE;
    if (misaligned({q, k, q_out, k_out}, elem_bytes(d->dtype)) || misaligned({gamma_q, gamma_k, pos}, 4) || misaligned({freq}, 8)) return PPO_ERR_ALIGN;
    QkArgs a = args(d, eps, q, k, gamma_q, gamma_k, pos, freq);
    a.qo = q_out;
    a.ko = k_out;
    return with_elem(d->dtype, [&](auto t) {
        return ppo_launch(qk_fwd_any_kernel<decltype(t)>, dim3(blocks_of(d)), dim3(256), 0, static_cast<cudaStream_t>(stream), a);
    });
}

extern "C" int ppo_qk_norm_rotate_bwd(const ppo_qk_norm_desc *d, float eps, const void *q, const void *k, const float *gamma_q, const float *gamma_k,
                                      const int32_t *pos, const double *freq, const void *dq_out, const void *dk_out, void *dq, void *dk,
                                      float *dgamma_q, float *dgamma_k, int accumulate, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    const bool params = dgamma_q || dgamma_k;
    if (!q || !k || !dq_out || !dk_out || !dq || !dk || (d->pairs > 0 && (!pos || !freq)) || !(eps >= 0.f) || (params && !workspace)) return PPO_ERR_INVALID_ARG;
    if ((dq == dq_out && d->ldq != d->ldqo) || (dk == dk_out && d->ldk != d->ldko)) return PPO_ERR_SHAPE;
    if (params && ws_bytes < ppo_qk_norm_rotate_workspace_bytes(d)) return PPO_ERR_SHAPE;
    if (misaligned({q, k, dq_out, dk_out, dq, dk}, elem_bytes(d->dtype)) || misaligned({gamma_q, gamma_k, dgamma_q, dgamma_k, pos}, 4) ||
        misaligned({freq}, 8) || misaligned({workspace}, 32))
        return PPO_ERR_ALIGN;
    QkArgs a = args(d, eps, q, k, gamma_q, gamma_k, pos, freq);
    a.dqo = dq_out;
    a.dko = dk_out;
    a.dq = dq;
    a.dk = dk;
    a.part = params ? static_cast<float *>(workspace) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int blocks = blocks_of(d);
    PPO_TRY(with_elem(d->dtype, [&](auto t) { return ppo_launch(qk_bwd_any_kernel<decltype(t)>, dim3(blocks), dim3(256), 0, st, a); }));
    return params ? ppo_param_sum(a.part, blocks, {{dgamma_q, dgamma_k, nullptr}, {d->d, d->d, 0}}, accumulate, st) : PPO_OK;
}
