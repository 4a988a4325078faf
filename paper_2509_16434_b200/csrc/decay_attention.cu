// Linear attention with a decay for each head: outputs, gradients, single steps.
//
// Outputs and all three gradients are one recurrence over the rows of a head, forwards or backwards in time, with a state
// M [R][C] and operands a, x [R], b [C]:
//   M <- lambda M + a b^T,   out = x^T M
//   o:  a = k, b = v,  x = q             dq: a = v,  b = k, x = do   (M = S^T)
//   dv: a = q, b = do, x = k, backwards  dk: a = do, b = q, x = v, backwards (M = dS^T)
// A set done flag empties M between that step and the one behind it.  Backwards, the decay is applied behind a step instead of
// in front of it: the gradient of the state that is left enters the last step undecayed, that of the state that came in
// leaves the first one decayed.
#include "elem.cuh"

namespace {

struct Sweep {
    const void *a, *b, *x;
    void *out;                     // type of the operands; heads that share one write theirs in 32 bits to `shared` instead
    float *shared;                 // [T * Be][heads][C]
    long long lda, ldb, ldx, ldo;  // elements from row to row
    int share_a, share_b, share_x; // heads per head of the operand
    const float *decay;
    const uint8_t *done;
    const float *m_in;
    float *m_out;
    long long state, stride_r, stride_c;  // elements of a state, from row to row and from column to column
    int T, Be, heads, R, C;
    float a_scale, out_scale;
    int reverse;
    int seg_len, nseg;   // steps per segment of the sequence (nseg == 1: all)
    float *seg;          // [nseg][Be * heads][R * C]: what each segment adds to a state, then what each starts from
};

constexpr int kTokens = 16, kCols = 32, kSlices = 4;

// One block: 32 columns of one head's state (a column per lane, R / 4 rows per warp) over one segment.
// STATE: only what the segment leaves behind, from an empty state.
template <typename T, int KS, bool STATE>
__global__ void __launch_bounds__(128) sweep_kernel(Sweep s) {
    grid_wait();
    constexpr int RP = KS * kSlices;
    __shared__ __align__(16) float ta[kTokens][RP], tx[kTokens][RP], tb[kTokens][kCols], part[kSlices][kTokens][kCols];
    __shared__ uint8_t gate[kTokens];
    const int lane = threadIdx.x % 32, w = threadIdx.x / 32;
    const int ncol = (s.C + kCols - 1) / kCols, c0 = blockIdx.x % ncol * kCols, c = c0 + lane;
    const int eh = blockIdx.x / ncol, e = eh / s.heads, h = eh % s.heads;
    const int seg = blockIdx.y;
    const float lam = s.decay[h];
    const T *A = static_cast<const T *>(s.a) + (long long)(h / s.share_a) * s.R;
    const T *B = static_cast<const T *>(s.b) + (long long)(h / s.share_b) * s.C;
    const T *X = static_cast<const T *>(s.x) + (long long)(h / s.share_x) * s.R;
    float M[KS];
    // this thread's element of row r of the state lies at r * sr + sc
    const long long sr = s.nseg > 1 ? s.C : s.stride_r, sc = s.nseg > 1 ? c : c * s.stride_c;
    const float *in = s.nseg > 1 ? s.seg + ((size_t)seg * s.Be * s.heads + eh) * s.R * s.C : s.m_in ? s.m_in + eh * s.state : nullptr;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int r = w * KS + i;
        M[i] = !STATE && in && r < s.R && c < s.C ? in[r * sr + sc] : 0.f;
    }
    const int n0 = seg * s.seg_len, n1 = min(n0 + s.seg_len, s.T);
    for (int n = n0; n < n1; n += kTokens) {
        const int cnt = min(kTokens, n1 - n);
        __syncthreads();
        for (int i = threadIdx.x; i < kTokens * RP; i += 128) {
            const int j = i / RP, r = i % RP;
            const int t = s.reverse ? s.T - 1 - (n + j) : n + j;
            const bool ok = j < cnt && r < s.R;
            const long long row = (long long)t * s.Be + e;
            ta[j][r] = ok ? to_f32(A[row * s.lda + r]) * s.a_scale : 0.f;
            if (!STATE) tx[j][r] = ok ? to_f32(X[row * s.ldx + r]) : 0.f;
        }
        for (int i = threadIdx.x; i < kTokens * kCols; i += 128) {
            const int j = i / kCols, k = i % kCols;
            const int t = s.reverse ? s.T - 1 - (n + j) : n + j;
            tb[j][k] = j < cnt && c0 + k < s.C ? to_f32(B[((long long)t * s.Be + e) * s.ldb + c0 + k]) : 0.f;
        }
        if (threadIdx.x < cnt) {
            const int t = s.reverse ? s.T - 1 - (n + threadIdx.x) : n + threadIdx.x;
            gate[threadIdx.x] = s.done && s.done[(long long)t * s.Be + e];
        }
        __syncthreads();
        for (int j = 0; j < cnt; ++j) {
            const float b = tb[j][lane];
            const bool empty = gate[j];
            float acc = 0.f;
            if (s.reverse && empty) {
#pragma unroll
                for (int i = 0; i < KS; ++i) M[i] = 0.f;
            }
            const float before = s.reverse ? 1.f : lam, after = s.reverse ? lam : 1.f;
#pragma unroll
            for (int i = 0; i < KS; i += 4) {
                const float4 a = *reinterpret_cast<const float4 *>(&ta[j][w * KS + i]);
                M[i] = fmaf(before, M[i], a.x * b);
                M[i + 1] = fmaf(before, M[i + 1], a.y * b);
                M[i + 2] = fmaf(before, M[i + 2], a.z * b);
                M[i + 3] = fmaf(before, M[i + 3], a.w * b);
                if constexpr (!STATE) {
                    const float4 x = *reinterpret_cast<const float4 *>(&tx[j][w * KS + i]);
                    acc = fmaf(x.x, M[i], acc);
                    acc = fmaf(x.y, M[i + 1], acc);
                    acc = fmaf(x.z, M[i + 2], acc);
                    acc = fmaf(x.w, M[i + 3], acc);
                }
            }
            if (s.reverse) {
#pragma unroll
                for (int i = 0; i < KS; ++i) M[i] *= after;
            } else if (empty) {
#pragma unroll
                for (int i = 0; i < KS; ++i) M[i] = 0.f;
            }
            if constexpr (!STATE) part[w][j][lane] = acc;
        }
        if constexpr (!STATE) {
            __syncthreads();
            for (int i = threadIdx.x; i < cnt * kCols; i += 128) {
                const int j = i / kCols, k = i % kCols;
                if (c0 + k >= s.C) continue;
                const int t = s.reverse ? s.T - 1 - (n + j) : n + j;
                const long long row = (long long)t * s.Be + e;
                const float v = s.out_scale * ((part[0][j][k] + part[1][j][k]) + (part[2][j][k] + part[3][j][k]));
                if (s.shared) s.shared[(row * s.heads + h) * s.C + c0 + k] = v;
                else static_cast<T *>(s.out)[row * s.ldo + (long long)h * s.C + c0 + k] = from_f32<T>(v);
            }
        }
    }
    float *out = STATE ? s.seg + ((size_t)seg * s.Be * s.heads + eh) * s.R * s.C : s.nseg > 1 || !s.m_out ? nullptr : s.m_out + eh * s.state;
    if (out && c < s.C) {
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const int r = w * KS + i;
            if (r < s.R) out[r * sr + sc] = M[i];
        }
    }
}

// decay ** n
__device__ __forceinline__ float power(float log2_decay, int n) { return n == 0 ? 1.f : exp2f((float)n * log2_decay); }

// What each segment starts from, in place of what it adds, and the state that is left.
__global__ void __launch_bounds__(256) segments_kernel(Sweep s) {
    grid_wait();
    __shared__ int reset;
    const int eh = blockIdx.x, e = eh / s.heads, h = eh % s.heads;
    const int i = blockIdx.y * 256 + threadIdx.x;  // element r * C + c
    const bool on = i < s.R * s.C;
    const long long at = on ? (i / s.C) * s.stride_r + (i % s.C) * s.stride_c : 0;
    const float l2 = log2f(s.decay[h]);
    float m = on && s.m_in ? s.m_in[eh * s.state + at] : 0.f;
    for (int seg = 0; seg < s.nseg; ++seg) {
        const int n0 = seg * s.seg_len, n1 = min(n0 + s.seg_len, s.T);
        __syncthreads();
        if (threadIdx.x == 0) reset = 0;
        __syncthreads();
        if (s.done) {
            bool any = false;
            for (int n = n0 + threadIdx.x; n < n1; n += 256) any |= s.done[(long long)(s.reverse ? s.T - 1 - n : n) * s.Be + e] != 0;
            if (any) reset = 1;
        }
        __syncthreads();
        if (on) {
            float *p = s.seg + ((size_t)seg * s.Be * s.heads + eh) * s.R * s.C + i;
            const float add = *p;
            *p = m;
            m = reset ? add : fmaf(power(l2, n1 - n0), m, add);
        }
    }
    if (on && s.m_out) s.m_out[eh * s.state + at] = m;
}

// Gradient of a shared head: the sum of those of its query heads.
template <typename T>
__global__ void __launch_bounds__(256) shared_sum_kernel(const float *part, T *out, long long ldo, long long rows, int kv_heads, int share, int C) {
    grid_wait();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / (kv_heads * C);
    if (row >= rows) return;
    const int at = (int)(i % (kv_heads * C)), g = at / C, c = at % C;
    const float *p = part + (row * kv_heads + g) * share * C + c;
    float v = 0.f;
    for (int k = 0; k < share; ++k) v += p[k * C];
    out[row * ldo + at] = from_f32<T>(v);
}

// One step of one head of one env per block: thread (g, l) holds columns VEC l.. of the rows g, g + groups, ...; the state
// goes through once, eight loads of a thread in flight.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) step_kernel(const T *q, const T *k, const T *v, T *o, const float *decay, const uint8_t *start, float *state,
                                                   long long ldq, long long ldk, long long ldv, long long ldo, int heads, int share, int dk, int dv,
                                                   float scale) {
    grid_wait();
    __shared__ float tq[128], tk[128], part[256 * VEC];
    const int e = blockIdx.x / heads, h = blockIdx.x % heads;
    const int lanes = dv / VEC, groups = 256 / lanes, g = threadIdx.x / lanes, c = threadIdx.x % lanes * VEC;
    float *S = state + (size_t)blockIdx.x * dk * dv + c;
    const bool on = g < groups, empty = start && start[e];
    const float lam = decay[h];
    for (int i = threadIdx.x; i < dk; i += 256) {
        tq[i] = to_f32(q[e * ldq + (long long)h * dk + i]) * scale;
        tk[i] = to_f32(k[e * ldk + (long long)(h / share) * dk + i]);
    }
    float val[VEC], acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        val[i] = on ? to_f32(v[e * ldv + (long long)(h / share) * dv + c + i]) : 0.f;
        acc[i] = 0.f;
    }
    bool first = true;
    for (int r0 = g; r0 < dk || first; r0 += 8 * groups) {
        float s[8][VEC];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = r0 + j * groups;
            const bool ok = on && r < dk && !empty;
            if constexpr (VEC == 4) {
                const float4 f = ok ? *reinterpret_cast<const float4 *>(S + (size_t)r * dv) : make_float4(0.f, 0.f, 0.f, 0.f);
                s[j][0] = f.x, s[j][1] = f.y, s[j][2] = f.z, s[j][3] = f.w;
            } else {
                s[j][0] = ok ? S[(size_t)r * dv] : 0.f;
            }
        }
        if (first) __syncthreads();
        first = false;
        if (!on) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = r0 + j * groups;
            if (r >= dk) break;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s[j][i] = fmaf(lam, s[j][i], tk[r] * val[i]);
                acc[i] = fmaf(tq[r], s[j][i], acc[i]);
            }
            if constexpr (VEC == 4) *reinterpret_cast<float4 *>(S + (size_t)r * dv) = make_float4(s[j][0], s[j][1], s[j][2], s[j][3]);
            else S[(size_t)r * dv] = s[j][0];
        }
    }
    if (on) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[g * dv + c + i] = acc[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < dv; i += 256) {
        float sum = 0.f;
        for (int j = 0; j < groups; ++j) sum += part[j * dv + i];
        o[e * ldo + (long long)h * dv + i] = from_f32<T>(sum);
    }
}

constexpr int kSegment = 256;

// Segments a sequence is cut into: as many as give the GPU two blocks per SM, none shorter than 256 steps.
int segments(const ppo_decay_attention_desc *d, int *len) {
    const long long blocks = (long long)d->Be * d->heads;
    int n = (int)((2 * 148 + blocks - 1) / blocks);
    const int most = ppo_cdiv(d->T, kSegment);
    if (n > most) n = most;
    const int per = ppo_cdiv(ppo_cdiv(d->T, n), 64) * 64;
    *len = per;
    return ppo_cdiv(d->T, per);
}

int check(const ppo_decay_attention_desc *d) {
    if (!d || d->T <= 0 || d->Be <= 0 || d->heads <= 0 || d->kv_heads <= 0 || d->dk <= 0 || d->dv <= 0) return PPO_ERR_INVALID_ARG;
    if (d->dtype != PPO_F32 && d->dtype != PPO_BF16) return PPO_ERR_INVALID_ARG;
    if (!(d->scale > -3.0e38f && d->scale < 3.0e38f)) return PPO_ERR_INVALID_ARG;
    if (d->heads % d->kv_heads != 0) return PPO_ERR_SHAPE;
    if (d->dk > 128 || d->dv > 128) return PPO_ERR_UNSUPPORTED;
    if ((long long)d->T * d->Be > 0x7fffffffll || (long long)d->Be * d->heads > 0x1fffffffll) return PPO_ERR_UNSUPPORTED;
    if (d->ldq < (int64_t)d->heads * d->dk || d->ldk < (int64_t)d->kv_heads * d->dk || d->ldv < (int64_t)d->kv_heads * d->dv ||
        d->ldo < (int64_t)d->heads * d->dv)
        return PPO_ERR_SHAPE;
    return PPO_OK;
}

size_t seg_floats(const ppo_decay_attention_desc *d) {
    int len;
    const int n = segments(d, &len);
    return n > 1 ? (size_t)n * d->Be * d->heads * d->dk * d->dv : 0;
}
size_t shared_floats(const ppo_decay_attention_desc *d) {
    return d->heads != d->kv_heads ? (size_t)d->T * d->Be * d->heads * (d->dk > d->dv ? d->dk : d->dv) : 0;
}

template <typename T, bool STATE>
int sweep_launch(const Sweep &s, cudaStream_t st) {
    const dim3 grid(ppo_cdiv(s.C, kCols) * s.Be * s.heads, s.nseg);
    if (s.R <= 32) return ppo_launch(sweep_kernel<T, 8, STATE>, grid, dim3(128), 0, st, s);
    if (s.R <= 64) return ppo_launch(sweep_kernel<T, 16, STATE>, grid, dim3(128), 0, st, s);
    return ppo_launch(sweep_kernel<T, 32, STATE>, grid, dim3(128), 0, st, s);
}
template <typename T>
int sweep(const Sweep &s, cudaStream_t st) {
    if (s.nseg > 1) {
        PPO_TRY(sweep_launch<T, true>(s, st));
        PPO_TRY(ppo_launch(segments_kernel, dim3(s.Be * s.heads, ppo_cdiv((long long)s.R * s.C, 256)), dim3(256), 0, st, s));
    }
    return sweep_launch<T, false>(s, st);
}

Sweep sweep_of(const ppo_decay_attention_desc *d, const float *decay, const uint8_t *done, float *seg) {
    Sweep s = {};
    s.decay = decay;
    s.done = done;
    s.state = (long long)d->dk * d->dv;
    s.T = d->T;
    s.Be = d->Be;
    s.heads = d->heads;
    s.a_scale = s.out_scale = 1.f;
    s.share_a = s.share_b = s.share_x = 1;
    s.nseg = segments(d, &s.seg_len);
    s.seg = seg;
    return s;
}
// M [dk][dv], the state as it is stored, or M [dv][dk]
void plain_state(Sweep *s, const ppo_decay_attention_desc *d) {
    s->R = d->dk;
    s->C = d->dv;
    s->stride_r = d->dv;
    s->stride_c = 1;
}
void turned_state(Sweep *s, const ppo_decay_attention_desc *d) {
    s->R = d->dv;
    s->C = d->dk;
    s->stride_r = 1;
    s->stride_c = d->dv;
}

bool misaligned(std::initializer_list<const void *> ps, size_t a) {
    for (const void *p : ps)
        if (!ppo_aligned(p, a)) return true;
    return false;
}

}  // namespace

extern "C" size_t ppo_decay_attention_workspace_bytes(const ppo_decay_attention_desc *d, int backward) {
    if (check(d) != PPO_OK) return 0;
    return (seg_floats(d) + (backward ? shared_floats(d) : 0)) * sizeof(float);
}

extern "C" int ppo_decay_attention_fwd(const ppo_decay_attention_desc *d, const void *q, const void *k, const void *v, const float *decay,
                                       const uint8_t *done, const float *state_in, void *o, float *state_out, void *workspace, size_t ws_bytes,
                                       void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_decay_attention_workspace_bytes(d, 0);
    if (!q || !k || !v || !decay || !o || (need > 0 && !workspace)) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({q, k, v, o}, elem_bytes(d->dtype)) || misaligned({decay}, 4) || misaligned({state_in, state_out, workspace}, 16)) return PPO_ERR_ALIGN;
    Sweep s = sweep_of(d, decay, done, static_cast<float *>(workspace));
    plain_state(&s, d);
    s.a = k, s.lda = d->ldk, s.b = v, s.ldb = d->ldv, s.x = q, s.ldx = d->ldq, s.out = o, s.ldo = d->ldo;
    s.share_a = s.share_b = d->heads / d->kv_heads;
    s.out_scale = d->scale;
    s.m_in = state_in;
    s.m_out = state_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d->dtype == PPO_F32 ? sweep<float>(s, st) : sweep<bf16>(s, st);
}

extern "C" int ppo_decay_attention_bwd(const ppo_decay_attention_desc *d, const void *q, const void *k, const void *v, const float *decay,
                                       const uint8_t *done, const float *state_in, const void *d_o, const float *dstate_out, void *dq, void *dk,
                                       void *dv, float *dstate_in, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_decay_attention_workspace_bytes(d, 1);
    if (!q || !k || !v || !decay || !d_o || !dq || !dk || !dv || (need > 0 && !workspace)) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({q, k, v, d_o, dq, dk, dv}, elem_bytes(d->dtype)) || misaligned({decay}, 4) ||
        misaligned({state_in, dstate_out, dstate_in, workspace}, 16))
        return PPO_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int share = d->heads / d->kv_heads;
    float *seg = static_cast<float *>(workspace), *part = share > 1 ? seg + seg_floats(d) : nullptr;
    const long long rows = (long long)d->T * d->Be;
    return [&](auto run) { return d->dtype == PPO_F32 ? run(float{}) : run(bf16{}); }([&](auto t) -> int {
        using T = decltype(t);
        Sweep s = sweep_of(d, decay, done, seg);
        turned_state(&s, d);
        s.a = v, s.lda = d->ldv, s.b = k, s.ldb = d->ldk, s.x = d_o, s.ldx = d->ldo, s.out = dq, s.ldo = d->ldq;
        s.share_a = s.share_b = share;
        s.out_scale = d->scale;
        s.m_in = state_in;
        PPO_TRY(sweep<T>(s, st));
        for (int key = 1; key >= 0; --key) {  // dk, then dv, which leaves the gradient of the state that came in
            s = sweep_of(d, decay, done, seg);
            s.reverse = 1;
            s.share_x = share;
            s.m_in = dstate_out;
            s.shared = part;
            T *out = static_cast<T *>(key ? dk : dv);
            if (key) {
                turned_state(&s, d);
                s.a = d_o, s.lda = d->ldo, s.b = q, s.ldb = d->ldq, s.x = v, s.ldx = d->ldv, s.ldo = d->ldk;
            } else {
                plain_state(&s, d);
                s.a = q, s.lda = d->ldq, s.b = d_o, s.ldb = d->ldo, s.x = k, s.ldx = d->ldk, s.ldo = d->ldv;
                s.m_out = dstate_in;
            }
            s.a_scale = d->scale;
            s.out = out;
            PPO_TRY(sweep<T>(s, st));
            if (part)
                PPO_TRY(ppo_launch(shared_sum_kernel<T>, dim3(ppo_cdiv(rows * d->kv_heads * s.C, 256)), dim3(256), 0, st, (const float *)part, out, s.ldo,
                                   rows, d->kv_heads, share, s.C));
        }
        return PPO_OK;
    });
}

extern "C" int ppo_decay_attention_step(const ppo_decay_attention_desc *d, const void *q, const void *k, const void *v, const float *decay,
                                        const uint8_t *start, float *state, void *o, void *stream) {
    PPO_TRY(check(d));
    if (d->T != 1) return PPO_ERR_SHAPE;
    if (!q || !k || !v || !decay || !state || !o) return PPO_ERR_INVALID_ARG;
    if (misaligned({q, k, v, o}, elem_bytes(d->dtype)) || misaligned({decay}, 4) || misaligned({state}, 16)) return PPO_ERR_ALIGN;
    return [&](auto run) { return d->dtype == PPO_F32 ? run(float{}) : run(bf16{}); }([&](auto t) -> int {
        using T = decltype(t);
        auto *fn = d->dv % 4 == 0 ? step_kernel<T, 4> : step_kernel<T, 1>;
        return ppo_launch(fn, dim3(d->Be * d->heads), dim3(256), 0, static_cast<cudaStream_t>(stream), static_cast<const T *>(q), static_cast<const T *>(k),
                          static_cast<const T *>(v), static_cast<T *>(o), decay, start, state, (long long)d->ldq, (long long)d->ldk, (long long)d->ldv,
                          (long long)d->ldo, (int)d->heads, (int)(d->heads / d->kv_heads), (int)d->dk, (int)d->dv, d->scale);
    });
}
