// Log-probabilities of tokens, and the clipped policy loss over a vocabulary with its gradient.
#include "elem.cuh"

namespace {

struct TokenArgs {
    const void *logits;
    const int32_t *tokens;
    long long ld, ld_grad;
    int rows, vocab;
    float scale;
    float *logp, *entropy;
    // the loss
    const float *old, *ref, *adv, *weight;
    void *grad;
    float clip_low, clip_high, kl_coef, ent_coef, grad_scale, inv_total;
    float *terms;  // [5][rows]
};

struct RowStat {
    float top, sum, xe;  // max, sum of e = exp(x - top), sum of e (x - top)
};
__device__ __forceinline__ RowStat merge(RowStat a, RowStat b) {
    if (b.top > a.top) {
        const RowStat t = a;
        a = b;
        b = t;
    }
    if (b.top == -INFINITY) return a;  // nothing in it
    const float d = b.top - a.top, f = expf(d);
    if (f > 0.f) {
        a.xe += f * (b.xe + d * b.sum);
        a.sum += f * b.sum;
    }
    return a;
}

constexpr int kRowThreads = 256;

template <typename T, bool LOSS>
__global__ void __launch_bounds__(kRowThreads) token_row_kernel(TokenArgs a) {
    grid_wait();
    __shared__ RowStat part[kRowThreads / 32];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T *x = static_cast<const T *>(a.logits) + (long long)row * a.ld;
    T *g = LOSS ? static_cast<T *>(a.grad) + (long long)row * a.ld_grad : nullptr;
    const int token = a.tokens[row];
    const float w = LOSS && a.weight ? a.weight[row] : 1.f;
    const bool out = token < 0 || token >= a.vocab || w == 0.f;
    RowStat s = {-INFINITY, 0.f, 0.f};
    if (!out) {
        float top = -INFINITY;
        for (int j = tid; j < a.vocab; j += kRowThreads) top = fmaxf(top, to_f32(x[j]) * a.scale);
        s.top = top;
        for (int j = tid; j < a.vocab; j += kRowThreads) {
            const float d = to_f32(x[j]) * a.scale - top, e = top == -INFINITY ? 0.f : expf(d);
            s.sum += e;
            if (e > 0.f) s.xe += e * d;
        }
    }
    for (int o = 16; o > 0; o >>= 1) {
        RowStat t;
        t.top = __shfl_xor_sync(0xffffffffu, s.top, o);
        t.sum = __shfl_xor_sync(0xffffffffu, s.sum, o);
        t.xe = __shfl_xor_sync(0xffffffffu, s.xe, o);
        s = merge(s, t);
    }
    if (tid % 32 == 0) part[tid / 32] = s;
    __syncthreads();
    s = part[0];
    for (int i = 1; i < kRowThreads / 32; ++i) s = merge(s, part[i]);
    const bool empty = s.top == -INFINITY;
    const float log_sum = logf(s.sum);
    float logp = out ? 0.f : empty ? -INFINITY : to_f32(x[token]) * a.scale - s.top - log_sum;
    const float H = out || empty ? 0.f : log_sum - s.xe / s.sum;
    if constexpr (!LOSS) {
        if (tid == 0) {
            a.logp[row] = logp;
            if (a.entropy) a.entropy[row] = H;
        }
        return;
    }
    const bool skip = out || empty;
    float dl = 0.f, share = 0.f;
    if (!skip) {
        const float ratio = expf(logp - a.old[row]), adv = a.adv[row];
        const float lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
        const float free_ = ratio * adv, held = fminf(fmaxf(ratio, lo), hi) * adv;
        float kl = 0.f;
        dl = free_ <= held ? -free_ : 0.f;
        if (a.ref) {
            const float d = a.ref[row] - logp, m = expm1f(d);
            kl = m - d;
            dl -= a.kl_coef * m;
        }
        share = w * a.inv_total;
        if (tid == 0) {
            const float t[5] = {-fminf(free_, held), kl, H, a.old[row] - logp, ratio < lo || ratio > hi ? 1.f : 0.f};
            for (int i = 0; i < 5; ++i) a.terms[(size_t)i * a.rows + row] = share * t[i];
        }
    } else if (tid == 0) {
        for (int i = 0; i < 5; ++i) a.terms[(size_t)i * a.rows + row] = 0.f;
        logp = 0.f;
    }
    if (tid == 0 && a.logp) a.logp[row] = logp;
    __syncthreads();  // the gradient may take the place of the logits: all have read x[token]
    const float inv = 1.f / s.sum, f = share * a.grad_scale * a.scale;
    for (int j = tid; j < a.vocab; j += kRowThreads) {
        float v = 0.f;
        if (!skip) {
            const float d = to_f32(x[j]) * a.scale - s.top, p = expf(d) * inv;
            v = -dl * p;
            if (p > 0.f) v += a.ent_coef * p * (d - log_sum + H);
            if (j == token) v += dl;
            v *= f;
        }
        g[j] = from_f32<T>(v);
    }
}

// Sums of the rows' terms in a fixed order, one block per term.
__global__ void __launch_bounds__(256) token_sum_kernel(const float *terms, int rows, float *out, int accumulate) {
    grid_wait();
    __shared__ double part[256];
    double s = 0;
    for (int i = threadIdx.x; i < rows; i += 256) s += terms[(size_t)blockIdx.x * rows + i];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if (threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) out[blockIdx.x] = (float)(part[0] + (accumulate ? (double)out[blockIdx.x] : 0.));
}

int check(const ppo_token_desc *d) {
    if (!d || d->rows <= 0 || d->vocab <= 0 || !(d->scale > 0.f) || d->scale > 3.0e38f) return PPO_ERR_INVALID_ARG;
    if (d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->ld < d->vocab) return PPO_ERR_SHAPE;
    return PPO_OK;
}

}  // namespace

extern "C" size_t ppo_token_loss_workspace_bytes(const ppo_token_desc *d) {
    return check(d) == PPO_OK ? (size_t)d->rows * 5 * sizeof(float) : 0;
}

extern "C" int ppo_token_logp(const ppo_token_desc *d, const void *logits, const int32_t *tokens, float *logp, float *entropy, void *stream) {
    PPO_TRY(check(d));
    if (!logits || !tokens || !logp) return PPO_ERR_INVALID_ARG;
    if (!ppo_aligned(logits, elem_bytes(d->dtype)) || !ppo_aligned(tokens, 4) || !ppo_aligned(logp, 4) || !ppo_aligned(entropy, 4)) return PPO_ERR_ALIGN;
    TokenArgs a = {};
    a.logits = logits;
    a.tokens = tokens;
    a.ld = d->ld;
    a.rows = d->rows;
    a.vocab = d->vocab;
    a.scale = d->scale;
    a.logp = logp;
    a.entropy = entropy;
    return with_elem(d->dtype, [&](auto t) {
        return ppo_launch(token_row_kernel<decltype(t), false>, dim3(d->rows), dim3(kRowThreads), 0, static_cast<cudaStream_t>(stream), a);
    });
}

extern "C" int ppo_token_loss_fwd_bwd(const ppo_token_desc *d, const ppo_token_loss_coef *c, const void *logits, const int32_t *tokens,
                                      const float *logp_old, const float *logp_ref, const float *adv, const float *weight, void *dlogits,
                                      int64_t ld_grad, float *logp_out, float *loss_out, int accumulate, void *workspace, size_t ws_bytes,
                                      void *stream) {
    PPO_TRY(check(d));
    if (!c || !logits || !tokens || !logp_old || !adv || !dlogits || !loss_out || !workspace) return PPO_ERR_INVALID_ARG;
    if (c->B_total <= 0 || !(c->clip_low >= 0.f) || !(c->clip_high >= 0.f)) return PPO_ERR_INVALID_ARG;
    if (ld_grad < d->vocab || (dlogits == logits && ld_grad != d->ld)) return PPO_ERR_SHAPE;
    if (ws_bytes < ppo_token_loss_workspace_bytes(d)) return PPO_ERR_SHAPE;
    const size_t e = elem_bytes(d->dtype);
    if (!ppo_aligned(logits, e) || !ppo_aligned(dlogits, e) || !ppo_aligned(workspace, 16)) return PPO_ERR_ALIGN;
    for (const void *p : {(const void *)tokens, (const void *)logp_old, (const void *)logp_ref, (const void *)adv, (const void *)weight,
                          (const void *)logp_out, (const void *)loss_out})
        if (!ppo_aligned(p, 4)) return PPO_ERR_ALIGN;
    TokenArgs a = {};
    a.logits = logits;
    a.tokens = tokens;
    a.ld = d->ld;
    a.ld_grad = ld_grad;
    a.rows = d->rows;
    a.vocab = d->vocab;
    a.scale = d->scale;
    a.logp = logp_out;
    a.old = logp_old;
    a.ref = logp_ref;
    a.adv = adv;
    a.weight = weight;
    a.grad = dlogits;
    a.clip_low = c->clip_low;
    a.clip_high = c->clip_high;
    a.kl_coef = c->kl_coef;
    a.ent_coef = c->ent_coef;
    a.grad_scale = c->grad_scale;
    a.inv_total = 1.f / (float)c->B_total;
    a.terms = static_cast<float *>(workspace);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    PPO_TRY(with_elem(d->dtype, [&](auto t) {
        return ppo_launch(token_row_kernel<decltype(t), true>, dim3(d->rows), dim3(kRowThreads), 0, st, a);
    }));
    return ppo_launch(token_sum_kernel, dim3(5), dim3(256), 0, st, (const float *)a.terms, (int)d->rows, loss_out, accumulate);
}
