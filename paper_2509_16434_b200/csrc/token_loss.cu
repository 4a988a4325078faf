// Log-probabilities of tokens, and the clipped policy loss over a vocabulary with its gradient.
//
// One pass: a row of logits is read once into registers, its maximum, sum of exponentials and sum of exponentials times logits are
// taken there, and the gradient is written from there.  A row belongs to a warp, to a block, or to a cluster of up to eight blocks
// that exchange their sums through distributed shared memory, by the bytes of a row alone: who sums what, and so every bit of a row's
// results, depends neither on the other rows of a call nor on where the row lies, and the call that scores a token while acting gives
// what the loss gives (a ratio of exactly 1 in a first epoch).
//
// Sums, maxima and arithmetic in 32 bits; only the gradient is rounded, once.  4096 rows of 32000 bf16 logits with their gradient, a tenth of the
// rows left out: 160 to 165 us, 3.0 to 3.1 TB/s of the 498 MB that have to move.  26 instructions for each logit, two exponentials among them, at two blocks of 16 warps an SM,
// which is what 64 registers a thread leave: loads of one block run under the arithmetic of the other.  Rows in shared memory, three
// blocks: 157, and log-probabilities of 40 rows of 100003 in 12.1 us, not 11.2; blocks that stay and copy rows ahead: 175.
#include "elem.cuh"
#include "tcgen05.cuh"

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

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Of logits x: the largest, the sum of e = 2^d with d = (x - top) scale log2(e), and the sum of e d.
struct RowStat {
    float top, sum, xe;
};
// Every rounding is written out, so that all kernels round alike.
__device__ __forceinline__ RowStat merge(RowStat a, RowStat b, float c) {
    if (b.top > a.top) {
        const RowStat t = a;
        a = b;
        b = t;
    }
    if (b.top == -INFINITY) return a;  // nothing in it
    const float d = __fmul_rn(b.top - a.top, c), f = exp2f(d);
    if (!(f == 0.f)) {
        a.xe = fmaf(f, fmaf(d, b.sum, b.xe), a.xe);
        a.sum = fmaf(f, b.sum, a.sum);
    }
    return a;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Bytes s .. s + 15 of 32.
__device__ __forceinline__ uint4 window(uint4 lo, uint4 hi, int s) {
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (s & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (s & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const int bits = (s & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}

// Single elements, at the ends of a row.
template <typename T>
__device__ __forceinline__ uint4 load_some(const T *x, int n) {
    constexpr int N = Vec<T>::N;
    T e[N];  // all on their way at a time
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = i < n ? x[i] : from_f32<T>(-INFINITY);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(e[i]);
        } else {
            w[i] = *reinterpret_cast<const uint16_t *>(&e[2 * i]) | (uint32_t)*reinterpret_cast<const uint16_t *>(&e[2 * i + 1]) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store_some(T *g, uint4 v, int from, int to) {
#pragma unroll 1
    for (int i = from; i < to; ++i) {
        if constexpr (sizeof(T) == 4) {
            g[i] = __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
        } else {
            const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
            *reinterpret_cast<uint16_t *>(g + i) = (uint16_t)(w >> (16 * (i & 1)));
        }
    }
}

// Elements 16 / sizeof(T) j .. of a row that starts anywhere; minus infinity behind its end.  plain: it is aligned and has whole vectors.
template <typename T>
__device__ __forceinline__ Vec<T> load_row(const T *x, int vocab, int j, bool plain) {
    constexpr int N = Vec<T>::N;
    const int s = (int)(reinterpret_cast<uintptr_t>(x) & 15), first = j * N;
    Vec<T> v;
    if (plain || first >= vocab) {
        constexpr uint32_t none = sizeof(T) == 4 ? 0xFF800000u : std::is_same_v<T, bf16> ? 0xFF80FF80u : 0xFC00FC00u;
        v.raw = first < vocab ? *reinterpret_cast<const uint4 *>(x + first) : make_uint4(none, none, none, none);
    } else if (first + N <= vocab && s == 0) {
        v.raw = *reinterpret_cast<const uint4 *>(x + first);
    } else if (j > 0 && first + 2 * N <= vocab) {  // both aligned windows lie inside the row
        const uint4 *p = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(x) - s) + j;
        v.raw = window(p[0], p[1], s);
    } else {
        v.raw = load_some(x + first, vocab - first);
    }
    return v;
}

// Stores elements N j .. of a row that starts anywhere; the lanes of the warp hold consecutive j.  Where the row is not aligned,
// a lane writes the aligned 16 bytes that its first elements share with the last ones of the lane in front.
template <typename T>
__device__ __forceinline__ void store_row(T *g, int vocab, int j, const Vec<T> &v, bool plain) {
    constexpr int N = Vec<T>::N;
    if (plain) {
        if (j * N < vocab) *reinterpret_cast<uint4 *>(g + j * N) = v.raw;
        return;
    }
    const int s = (int)(reinterpret_cast<uintptr_t>(g) & 15), lane = threadIdx.x & 31, first = j * N;
    const bool full = first + N <= vocab;
    if (s == 0) {
        if (full) *reinterpret_cast<uint4 *>(g + first) = v.raw;
        else if (first < vocab) store_some(g + first, v.raw, 0, vocab - first);
        return;
    }
    uint4 prev;
    prev.x = __shfl_up_sync(0xffffffffu, v.raw.x, 1);
    prev.y = __shfl_up_sync(0xffffffffu, v.raw.y, 1);
    prev.z = __shfl_up_sync(0xffffffffu, v.raw.z, 1);
    prev.w = __shfl_up_sync(0xffffffffu, v.raw.w, 1);
    const int split = (16 - s) / (int)sizeof(T);  // elements in front of the next aligned address
    if (first >= vocab) return;
    if (lane > 0 && full) *(reinterpret_cast<uint4 *>(reinterpret_cast<uintptr_t>(g) - s) + j) = window(prev, v.raw, 16 - s);
    else store_some(g + first, v.raw, 0, min(split, vocab - first));
    if (lane == 31 || first + 2 * N > vocab) store_some(g + first, v.raw, split, min(N, vocab - first));
}

// The larger ones of two vectors' elements, and the largest of one's; a NaN gives way to a number.
template <typename T>
__device__ __forceinline__ uint32_t max_word(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    } else if constexpr (std::is_same_v<T, bf16>) {
        const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    } else {
        const __half2 m = __hmax2(*reinterpret_cast<__half2 *>(&a), *reinterpret_cast<__half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
}
template <typename T>
__device__ __forceinline__ uint4 max_of(uint4 a, uint4 b) {
    return make_uint4(max_word<T>(a.x, b.x), max_word<T>(a.y, b.y), max_word<T>(a.z, b.z), max_word<T>(a.w, b.w));
}
template <typename T>
__device__ __forceinline__ float largest(uint4 a) {
    Vec<T> v;
    float f[Vec<T>::N], m = -INFINITY;
    v.raw = a;
    v.get(f);
#pragma unroll
    for (int k = 0; k < Vec<T>::N; ++k) m = fmaxf(m, f[k]);
    return m;
}

// Keeps the compiler from holding the elements of a vector, unpacked, from one use to the next: there are registers for them packed only.
__device__ __forceinline__ void stay_packed(uint4 &v) { asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)); }

// What is said of a row besides its logits.
struct RowSaid {
    int token;
    float w, old, adv, ref;
    bool out;  // left out: nothing else of it counts
};
template <bool LOSS>
__device__ __forceinline__ RowSaid said_of(const TokenArgs &a, int row) {
    RowSaid r = {a.tokens[row], 1.f, 0.f, 0.f, 0.f, false};
    if (LOSS) {
        if (a.weight) r.w = a.weight[row];
        r.old = a.old[row];
        r.adv = a.adv[row];
        if (a.ref) r.ref = a.ref[row];
    }
    r.out = r.token < 0 || r.token >= a.vocab || r.w == 0.f;
    return r;
}

// The sums of the vectors that the WARPS warps of a row hold (thread t of them), of which this warp has `filled`; those behind them are
// minus infinity and would change nothing.  Their largest first: sums about one common value need no factors when they are joined.
template <typename T, int NV, int WARPS>
__device__ __forceinline__ RowStat stat_of(Vec<T> (&v)[NV], int filled, bool out, float c, int t, float (&part)[3][WARPS]) {
    constexpr int N = Vec<T>::N;
    RowStat r = {-INFINITY, 0.f, 0.f};
    if (!out) {
        uint4 most = v[0].raw;
#pragma unroll
        for (int i = 1; i < NV; ++i) most = max_of<T>(most, v[i].raw);
        r.top = largest<T>(most);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r.top = fmaxf(r.top, __shfl_xor_sync(0xffffffffu, r.top, o));
    if constexpr (WARPS > 1) {
        if (t % 32 == 0) part[0][t / 32] = r.top;
        __syncthreads();
        r.top = part[0][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) r.top = fmaxf(r.top, part[0][i]);
    }
    const float top = r.top == -INFINITY ? 0.f : r.top;
    if (!out) {
        const auto add = [&](Vec<T> &x) {
            float f[N];
            stay_packed(x.raw);
            x.get(f);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = __fmul_rn(f[k] - top, c), e = exp2_fast(d);
                r.sum += e;
                r.xe = fmaf(e, fmaxf(d, -150.f), r.xe);  // e is 0 from there on
            }
        };
        if (filled == NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) add(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < filled) add(v[i]);
        }
    }
    r.sum = warp_sum(r.sum);
    r.xe = warp_sum(r.xe);
    if constexpr (WARPS > 1) {
        if (t % 32 == 0) {
            part[1][t / 32] = r.sum;
            part[2][t / 32] = r.xe;
        }
        __syncthreads();
        r.sum = part[1][0];
        r.xe = part[2][0];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) {
            r.sum += part[1][i];
            r.xe += part[2][i];
        }
    }
    if (r.sum != r.sum) r.top = INFINITY;  // a NaN among numbers, or alone: the row's results are NaN
    return r;
}

// The gradient as e (alpha + beta d), and `hot` more at the token; skip: zeros.
struct RowGrad {
    float alpha, beta, hot;
    bool skip;
};
// A row's results from its sums; the first thread writes the scalars.
template <bool LOSS>
__device__ __forceinline__ RowGrad results(const TokenArgs &a, int row, const RowSaid &r, float xa, const RowStat &s, bool first) {
    const bool empty = s.top == -INFINITY;
    const float log_sum = logf(s.sum);
    float logp = r.out ? 0.f : empty ? -INFINITY : fmaf(xa - s.top, a.scale, -log_sum);
    const float H = r.out || empty ? 0.f : fmaf(-kLn2, s.xe / s.sum, log_sum);
    if constexpr (!LOSS) {
        if (first) {
            a.logp[row] = logp;
            if (a.entropy) a.entropy[row] = H;
        }
        return {};
    } else {
        const bool skip = r.out || empty;
        float dl = 0.f, share = 0.f, terms[5] = {};
        if (skip) {
            logp = 0.f;
        } else {
            const float ratio = expf(logp - r.old), lo = 1.f - a.clip_low, hi = 1.f + a.clip_high;
            // NaN is kept: it shows in gradient and sums
            const float free_ = ratio * r.adv, held = (ratio < lo ? lo : ratio > hi ? hi : ratio) * r.adv;
            dl = free_ > held ? 0.f : -free_;
            share = r.w * a.inv_total;
            terms[0] = -share * (free_ > held ? held : free_);
            if (a.ref) {
                const float d = r.ref - logp, m = expm1f(d);
                terms[1] = share * (m - d);
                dl -= a.kl_coef * m;
            }
            terms[2] = share * H;
            terms[3] = share * (r.old - logp);
            terms[4] = ratio < lo || ratio > hi ? share : 0.f;
        }
        if (first) {
#pragma unroll
            for (int i = 0; i < 5; ++i) a.terms[(size_t)i * a.rows + row] = terms[i];
            if (a.logp) a.logp[row] = logp;
        }
        const float f = share * a.grad_scale * a.scale, inv = f / s.sum;
        return {inv * fmaf(a.ent_coef, H - log_sum, -dl), inv * a.ent_coef * kLn2, f * dl, skip};
    }
}
// Of vector j.
template <typename T>
__device__ __forceinline__ Vec<T> grad_of(Vec<T> &v, int j, int token, float top, float c, const RowGrad &g) {
    constexpr int N = Vec<T>::N;
    float o[N];
    if (g.skip) {
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] = 0.f;
    } else {
        stay_packed(v.raw);
        v.get(o);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float d = __fmul_rn(o[k] - top, c);
            o[k] = exp2_fast(d) * fmaf(g.beta, fmaxf(d, -150.f), g.alpha);
        }
        if (token / N == j) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (token % N == k) o[k] += g.hot;
        }
    }
    Vec<T> r;
    r.set(o);
    return r;
}

// THREADS per row and block of a cluster, NV 16-byte vectors of each in registers; rows that are longer than the cluster's
// registers are read in pieces, and again for the gradient.
template <typename T, int THREADS, int NV, bool LOSS>
__global__ void __launch_bounds__(THREADS < 128 ? 128 : THREADS, THREADS == 512 ? 2 : 6) token_row_kernel(TokenArgs a, int cluster) {
    grid_wait();
    constexpr int N = Vec<T>::N, WARPS = THREADS / 32;
    __shared__ float part[3][WARPS];
    __shared__ RowStat whole[8];
    if (cluster > 1) tc::cluster_arrive();
    const int t = threadIdx.x % THREADS;
    const int rank = cluster > 1 ? blockIdx.x % cluster : 0;
    const int row = THREADS < 128 ? blockIdx.x * (128 / THREADS) + threadIdx.x / THREADS : blockIdx.x / cluster;
    if (row >= a.rows) return;  // a whole warp
    const T *x = static_cast<const T *>(a.logits) + (long long)row * a.ld;
    const bool plain = a.vocab % N == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    const RowSaid said = said_of<LOSS>(a, row);
    const float c = a.scale * kLog2e;
    const int step = THREADS * cluster, j0 = rank * THREADS + t, pieces = (a.vocab + N * NV * step - 1) / (N * NV * step);
    Vec<T> v[NV];
    RowStat s = {-INFINITY, 0.f, 0.f};
    const float xa = said.out ? 0.f : to_f32(x[said.token]);
    const auto load = [&](int p) {
        if (said.out) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = load_row(x, a.vocab, (p * NV + i) * step + j0, plain);
    };
    for (int p = 0; p < pieces; ++p) {
        load(p);
        if (WARPS > 1 && p > 0) __syncthreads();  // the sums of the piece before are read
        const int left = max(0, a.vocab - (p * NV * step + (j0 & ~31)) * N);  // elements from this warp's first vector on
        const RowStat r = stat_of<T, NV, WARPS>(v, min(NV, (left + N * step - 1) / (N * step)), said.out, c, t, part);
        s = p == 0 ? r : merge(s, r, c);
    }
    if constexpr (WARPS > 1) {
        if (cluster > 1) {
            tc::cluster_wait();  // all blocks of the cluster run
            if (t < cluster) {   // to each block of the cluster
                const uint32_t at = tc::in_cta(tc::smem_u32(&whole[rank]), t);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(s.top) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(s.sum) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(s.xe) : "memory");
            }
            tc::cluster_sync();
            s = whole[0];
            for (int i = 1; i < cluster; ++i) s = merge(s, whole[i], c);
        }
    }
    const RowGrad grad = results<LOSS>(a, row, said, xa, s, t == 0 && rank == 0);
    if constexpr (LOSS) {
        T *g = static_cast<T *>(a.grad) + (long long)row * a.ld_grad;
        const bool plain_g = a.vocab % N == 0 && (reinterpret_cast<uintptr_t>(g) & 15) == 0;
        __syncwarp();  // in place: all lanes have read their logits, and the token's
        for (int p = 0; p < pieces; ++p) {
            if (pieces > 1 && !grad.skip) load(p);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int j = (p * NV + i) * step + j0;
                if ((j & ~31) * N >= a.vocab) break;  // the same in all lanes
                store_row(g, a.vocab, j, grad_of(v[i], j, said.token, s.top, c, grad), plain_g);
            }
        }
    }
}

// Sums of the rows' terms in a fixed order, one block per term, eight loads of a thread in flight.
__global__ void __launch_bounds__(512) token_sum_kernel(const float *terms, int rows, float *out, int accumulate) {
    grid_wait();
    __shared__ double part[512];
    double s = 0;
#pragma unroll 8
    for (int i = threadIdx.x; i < rows; i += 512) s += terms[(size_t)blockIdx.x * rows + i];
    part[threadIdx.x] = s;
    __syncthreads();
    for (int o = 256; o > 0; o >>= 1) {
        if (threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) out[blockIdx.x] = (float)(part[0] + (accumulate ? (double)out[blockIdx.x] : 0.));
}

// A warp for rows of up to 4 KB, a block of 128 threads to 16 KB, of 512 to 64 KB, then clusters of 2, 4, 8 blocks (to 512 KB in
// registers): as few threads as hold the row, which meet at the fewest barriers.  Gradients, bf16: 32768 rows of 2048 91 us, by 128 threads
// 265; 8192 of 8192 86, by 512 threads 259; 4096 of 32000 160, by two blocks 312 (with a warp's empty vectors left out, since then, the
// larger ones lose less: 8192 rows of 9000 263 -> 168).
template <typename T, bool LOSS>
int launch_rows(const TokenArgs &a, cudaStream_t st) {
    const size_t bytes = (size_t)a.vocab * sizeof(T);
    if (bytes <= 4096) return ppo_launch(token_row_kernel<T, 32, 8, LOSS>, dim3(ppo_cdiv(a.rows, 4)), dim3(128), 0, st, a, 1);
    if (bytes <= 16384) return ppo_launch(token_row_kernel<T, 128, 8, LOSS>, dim3(a.rows), dim3(128), 0, st, a, 1);
    int n = 1;
    while (n < 8 && bytes > (size_t)n * 65536) n *= 2;
    return ppo_launch_cluster(token_row_kernel<T, 512, 8, LOSS>, n, dim3(a.rows * n), dim3(512), 0, st, a, n);
}

int check(const ppo_token_desc *d) {
    if (!d || d->rows <= 0 || d->vocab <= 0 || !(d->scale > 0.f) || d->scale > 1.0e38f) return PPO_ERR_INVALID_ARG;
    if (d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->ld < d->vocab) return PPO_ERR_SHAPE;
    if (d->rows > 0x7fffffff / 8 || d->vocab > 0x7fffffff / 2) return PPO_ERR_UNSUPPORTED;
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
        return launch_rows<decltype(t), false>(a, static_cast<cudaStream_t>(stream));
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
    if (!ppo_aligned(logits, e) || !ppo_aligned(dlogits, e) || !ppo_aligned(workspace, 32)) return PPO_ERR_ALIGN;
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
        return launch_rows<decltype(t), true>(a, st);
    }));
    return ppo_launch(token_sum_kernel, dim3(5), dim3(512), 0, st, (const float *)a.terms, (int)d->rows, loss_out, accumulate);
}
