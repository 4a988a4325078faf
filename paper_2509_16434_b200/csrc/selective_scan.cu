// Selective scan: states whose decay and input the data choose, and its gradients.
//
// A thread takes one channel of one env and goes through the steps; states, sums and arithmetic in 32 bits.
#include "elem.cuh"
#include "param_sum.cuh"

namespace {

constexpr int kMaxN = 64;

struct ScanArgs {
    const void *x, *dt, *B, *C, *z, *dy;
    const float *A, *D, *bias, *state_in, *dstate_out;
    const uint8_t *done, *start;
    void *y, *dx, *ddt, *dB, *dC, *dz;
    float *state_out, *dstate_in;
    float *hist, *back, *part;  // states and their gradients of every step [T][Be][C][N]; shares of parameters [Be][C N + C + C]
    long long ldx, lddt, ldb, ldc, ldz, ldy;
    int T, Be, channels, N, groups, softplus;
};

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.f) + log1pf(expf(-fabsf(v))); }

template <typename T>
__global__ void __launch_bounds__(128) scan_fwd_kernel(ScanArgs a, bool keep) {
    grid_wait();
    const int cols = (a.channels + 127) / 128, e = blockIdx.x / cols, c = blockIdx.x % cols * 128 + threadIdx.x, N = a.N;
    if (c >= a.channels) return;
    const int g = c / (a.channels / a.groups);
    const size_t at = ((size_t)e * a.channels + c) * N;
    float h[kMaxN];
    const bool empty = !a.state_in || (a.start && a.start[e]);
    for (int n = 0; n < N; ++n) h[n] = empty ? 0.f : a.state_in[at + n];
    for (int t = 0; t < a.T; ++t) {
        const long long row = (long long)t * a.Be + e;
        const float x = to_f32(static_cast<const T *>(a.x)[row * a.ldx + c]);
        float d = to_f32(static_cast<const T *>(a.dt)[row * a.lddt + c]) + (a.bias ? a.bias[c] : 0.f), y = 0.f;
        if (a.softplus) d = softplus(d);
        const T *B = static_cast<const T *>(a.B) + row * a.ldb + g * N, *C = static_cast<const T *>(a.C) + row * a.ldc + g * N;
        for (int n = 0; n < N; ++n) {
            h[n] = fmaf(expf(d * a.A[(size_t)c * N + n]), h[n], d * x * to_f32(B[n]));
            y = fmaf(to_f32(C[n]), h[n], y);
            if (keep) a.hist[((size_t)t * a.Be * a.channels) * N + at + n] = h[n];
        }
        if (a.y) {
            if (a.D) y = fmaf(a.D[c], x, y);
            if (a.z) {
                const float z = to_f32(static_cast<const T *>(a.z)[row * a.ldz + c]);
                y *= z * sigmoid(z);
            }
            static_cast<T *>(a.y)[row * a.ldy + c] = from_f32<T>(y);
        }
        if (a.done && a.done[row])
            for (int n = 0; n < N; ++n) h[n] = 0.f;
    }
    if (a.state_out)
        for (int n = 0; n < N; ++n) a.state_out[at + n] = h[n];
}

template <typename T>
__global__ void __launch_bounds__(128) scan_bwd_kernel(ScanArgs a) {
    grid_wait();
    const int cols = (a.channels + 127) / 128, e = blockIdx.x / cols, c = blockIdx.x % cols * 128 + threadIdx.x, N = a.N;
    if (c >= a.channels) return;
    const int gr = c / (a.channels / a.groups);
    const size_t at = ((size_t)e * a.channels + c) * N, step = (size_t)a.Be * a.channels * N;
    float g[kMaxN], dA[kMaxN], dD = 0.f, dbias = 0.f;
    for (int n = 0; n < N; ++n) {
        g[n] = a.dstate_out ? a.dstate_out[at + n] : 0.f;
        dA[n] = 0.f;
    }
    for (int t = a.T - 1; t >= 0; --t) {
        const long long row = (long long)t * a.Be + e;
        const float x = to_f32(static_cast<const T *>(a.x)[row * a.ldx + c]), raw = to_f32(static_cast<const T *>(a.dt)[row * a.lddt + c]) + (a.bias ? a.bias[c] : 0.f);
        const float d = a.softplus ? softplus(raw) : raw, dout = to_f32(static_cast<const T *>(a.dy)[row * a.ldy + c]);
        const T *B = static_cast<const T *>(a.B) + row * a.ldb + gr * N, *C = static_cast<const T *>(a.C) + row * a.ldc + gr * N;
        float z = 0.f, sz = 0.f, dy = dout, y = a.D ? a.D[c] * x : 0.f, s1 = 0.f, s2 = 0.f;
        if (a.z) {
            z = to_f32(static_cast<const T *>(a.z)[row * a.ldz + c]);
            sz = sigmoid(z);
            dy = dout * z * sz;
        }
        const bool reset = a.done && a.done[row], before = t > 0 && a.done && a.done[row - a.Be];
        for (int n = 0; n < N; ++n) {
            const float A = a.A[(size_t)c * N + n], f = expf(d * A), h = a.hist[t * step + at + n];
            const float last = before ? 0.f : t > 0 ? a.hist[(t - 1) * step + at + n] : a.state_in ? a.state_in[at + n] : 0.f;
            y = fmaf(to_f32(C[n]), h, y);
            g[n] = fmaf(to_f32(C[n]), dy, reset ? 0.f : g[n]);
            a.back[t * step + at + n] = g[n];
            s1 = fmaf(g[n], to_f32(B[n]), s1);
            g[n] *= f;
            const float q = g[n] * last;
            s2 = fmaf(q, A, s2);
            dA[n] = fmaf(q, d, dA[n]);
        }
        float dd = fmaf(x, s1, s2);
        if (a.softplus) dd *= sigmoid(raw);
        static_cast<T *>(a.dx)[row * a.ldx + c] = from_f32<T>(fmaf(d, s1, a.D ? a.D[c] * dy : 0.f));
        static_cast<T *>(a.ddt)[row * a.lddt + c] = from_f32<T>(dd);
        if (a.z) static_cast<T *>(a.dz)[row * a.ldz + c] = from_f32<T>(dout * y * (sz * fmaf(z, 1.f - sz, 1.f)));
        dD = fmaf(dy, x, dD);
        dbias += dd;
    }
    for (int n = 0; n < N; ++n)
        if (a.dstate_in) a.dstate_in[at + n] = g[n];
    float *part = a.part + (size_t)e * a.channels * (N + 2);
    for (int n = 0; n < N; ++n) part[(size_t)c * N + n] = dA[n];
    part[(size_t)a.channels * N + c] = dD;
    part[(size_t)a.channels * (N + 1) + c] = dbias;
}

// Sums over the channels of a group, for the gradients of B and C of one row.
template <typename T>
__global__ void __launch_bounds__(128) scan_shared_kernel(ScanArgs a) {
    grid_wait();
    const long long row = blockIdx.x;
    const int per = a.channels / a.groups;
    for (int i = threadIdx.x; i < a.groups * a.N; i += 128) {
        const int n = i % a.N, c0 = i / a.N * per;
        float sb = 0.f, sc = 0.f;
        for (int c = c0; c < c0 + per; ++c) {
            const size_t at = ((size_t)row * a.channels + c) * a.N + n;
            const float x = to_f32(static_cast<const T *>(a.x)[row * a.ldx + c]);
            float d = to_f32(static_cast<const T *>(a.dt)[row * a.lddt + c]) + (a.bias ? a.bias[c] : 0.f), dy = to_f32(static_cast<const T *>(a.dy)[row * a.ldy + c]);
            if (a.softplus) d = softplus(d);
            if (a.z) {
                const float z = to_f32(static_cast<const T *>(a.z)[row * a.ldz + c]);
                dy *= z * sigmoid(z);
            }
            sb = fmaf(a.back[at], d * x, sb);
            sc = fmaf(a.hist[at], dy, sc);
        }
        static_cast<T *>(a.dB)[row * a.ldb + i] = from_f32<T>(sb);
        static_cast<T *>(a.dC)[row * a.ldc + i] = from_f32<T>(sc);
    }
}

int check(const ppo_selective_scan_desc *d) {
    if (!d || d->T <= 0 || d->Be <= 0 || d->channels <= 0 || d->N <= 0 || d->groups <= 0) return PPO_ERR_INVALID_ARG;
    if (d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->channels % d->groups != 0) return PPO_ERR_SHAPE;
    if (d->N > kMaxN || (long long)d->T * d->Be > 0x7f000000ll || (long long)d->Be * d->channels > 0x1fffffffll) return PPO_ERR_UNSUPPORTED;
    const int64_t few = (int64_t)d->groups * d->N;
    if (d->ldx < d->channels || d->lddt < d->channels || d->ldz < d->channels || d->ldy < d->channels || d->ldb < few || d->ldc < few) return PPO_ERR_SHAPE;
    return PPO_OK;
}
bool misaligned(std::initializer_list<const void *> ps, size_t a) {
    for (const void *p : ps)
        if (!ppo_aligned(p, a)) return true;
    return false;
}

ScanArgs args(const ppo_selective_scan_desc *d, const void *x, const void *dt, const float *A, const void *B, const void *C, const float *D,
              const void *z, const float *bias) {
    ScanArgs a = {};
    a.x = x;
    a.dt = dt;
    a.A = A;
    a.B = B;
    a.C = C;
    a.D = D;
    a.z = z;
    a.bias = bias;
    a.ldx = d->ldx;
    a.lddt = d->lddt;
    a.ldb = d->ldb;
    a.ldc = d->ldc;
    a.ldz = d->ldz;
    a.ldy = d->ldy;
    a.T = d->T;
    a.Be = d->Be;
    a.channels = d->channels;
    a.N = d->N;
    a.groups = d->groups;
    a.softplus = d->softplus;
    return a;
}

}  // namespace

extern "C" size_t ppo_selective_scan_workspace_bytes(const ppo_selective_scan_desc *d, int backward) {
    if (check(d) != PPO_OK || !backward) return 0;
    return ((size_t)2 * d->T * d->Be * d->channels * d->N + (size_t)d->Be * d->channels * (d->N + 2)) * sizeof(float);
}

extern "C" int ppo_selective_scan_fwd(const ppo_selective_scan_desc *d, const void *x, const void *dt, const float *A, const void *B, const void *C,
                                      const float *D, const void *z, const float *dt_bias, const uint8_t *done, const float *state_in, void *y,
                                      float *state_out, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_selective_scan_workspace_bytes(d, 0);
    if (!x || !dt || !A || !B || !C || !y || (need > 0 && !workspace)) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({x, dt, B, C, z, y}, elem_bytes(d->dtype)) || misaligned({A, D, dt_bias}, 4) || misaligned({state_in, state_out}, 16) ||
        misaligned({workspace}, 32))
        return PPO_ERR_ALIGN;
    ScanArgs a = args(d, x, dt, A, B, C, D, z, dt_bias);
    a.done = done;
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    return with_elem(d->dtype, [&](auto t) {
        return ppo_launch(scan_fwd_kernel<decltype(t)>, dim3(d->Be * ppo_cdiv(d->channels, 128)), dim3(128), 0, static_cast<cudaStream_t>(stream), a, false);
    });
}

extern "C" int ppo_selective_scan_bwd(const ppo_selective_scan_desc *d, const void *x, const void *dt, const float *A, const void *B, const void *C,
                                      const float *D, const void *z, const float *dt_bias, const uint8_t *done, const float *state_in, const void *dy,
                                      const float *dstate_out, void *dx, void *ddt, float *dA, void *dB, void *dC, float *dD, void *dz, float *ddt_bias,
                                      float *dstate_in, int accumulate, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_selective_scan_workspace_bytes(d, 1);
    if (!x || !dt || !A || !B || !C || !dy || !dx || !ddt || !dB || !dC || !z != !dz || !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({x, dt, B, C, z, dy, dx, ddt, dB, dC, dz}, elem_bytes(d->dtype)) || misaligned({A, D, dt_bias, dA, dD, ddt_bias}, 4) ||
        misaligned({state_in, dstate_out, dstate_in}, 16) || misaligned({workspace}, 32))
        return PPO_ERR_ALIGN;
    ScanArgs a = args(d, x, dt, A, B, C, D, z, dt_bias);
    const size_t steps = (size_t)d->T * d->Be * d->channels * d->N;
    a.done = done;
    a.state_in = state_in;
    a.dy = dy;
    a.dstate_out = dstate_out;
    a.dx = dx;
    a.ddt = ddt;
    a.dB = dB;
    a.dC = dC;
    a.dz = dz;
    a.dstate_in = dstate_in;
    a.hist = static_cast<float *>(workspace);
    a.back = a.hist + steps;
    a.part = a.back + steps;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    PPO_TRY(with_elem(d->dtype, [&](auto t) -> int {
        const dim3 grid(d->Be * ppo_cdiv(d->channels, 128));
        PPO_TRY(ppo_launch(scan_fwd_kernel<decltype(t)>, grid, dim3(128), 0, st, a, true));
        PPO_TRY(ppo_launch(scan_bwd_kernel<decltype(t)>, grid, dim3(128), 0, st, a));
        return ppo_launch(scan_shared_kernel<decltype(t)>, dim3(d->T * d->Be), dim3(128), 0, st, a);
    }));
    if (!dA && !dD && !ddt_bias) return PPO_OK;
    return ppo_param_sum(a.part, d->Be, {{dA, dD, ddt_bias}, {d->channels * d->N, d->channels, d->channels}}, accumulate, st);
}

extern "C" int ppo_selective_scan_step(const ppo_selective_scan_desc *d, const void *x, const void *dt, const float *A, const void *B, const void *C,
                                       const float *D, const void *z, const float *dt_bias, const uint8_t *start, float *state, void *y, void *stream) {
    PPO_TRY(check(d));
    if (d->T != 1) return PPO_ERR_SHAPE;
    if (!x || !dt || !A || !B || !C || !state || !y) return PPO_ERR_INVALID_ARG;
    if (misaligned({x, dt, B, C, z, y}, elem_bytes(d->dtype)) || misaligned({A, D, dt_bias}, 4) || misaligned({state}, 16)) return PPO_ERR_ALIGN;
    ScanArgs a = args(d, x, dt, A, B, C, D, z, dt_bias);
    a.start = start;
    a.state_in = state;
    a.y = y;
    a.state_out = state;
    return with_elem(d->dtype, [&](auto t) {
        return ppo_launch(scan_fwd_kernel<decltype(t)>, dim3(d->Be * ppo_cdiv(d->channels, 128)), dim3(128), 0, static_cast<cudaStream_t>(stream), a, false);
    });
}
