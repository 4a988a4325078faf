// Causal convolution of each channel along the steps of an env, with an activation, and its gradients.
//
// A thread takes V neighbouring channels over a run of steps of one env and keeps the last width - 1 inputs in registers: every input is
// read once (but for the width - 1 in front of a run) and every output written once.  Sums in 32 bits.
#include "elem.cuh"
#include "param_sum.cuh"

namespace {

struct ConvArgs {
    const void *x, *state_in, *dy, *dstate_out;
    void *y, *state_out, *dx, *dstate_in;
    const float *weight, *bias;
    const uint8_t *done;
    float *part;  // shares of the gradients of weight and bias, [parts][C * width + C]
    long long ldx, ldy;
    int T, Be, C, act, run, tiles;
};

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
__device__ __forceinline__ float activate(float z, int act) {
    return act == PPO_ACT_SILU ? z * sigmoid(z) : act == PPO_ACT_RELU ? (z < 0.f ? 0.f : z) : z;
}
__device__ __forceinline__ float grad_act(float z, int act) {
    if (act == PPO_ACT_SILU) {
        const float p = sigmoid(z);
        return p * fmaf(z, 1.f - p, 1.f);
    }
    return act == PPO_ACT_RELU && !(z > 0.f) ? 0.f : 1.f;
}

// V elements, aligned to all of them.
template <typename T, int V>
__device__ __forceinline__ void load(const T *p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = to_f32(*p);
    } else if constexpr (V * sizeof(T) == 16) {
        Vec<T> r;
        r.raw = *reinterpret_cast<const uint4 *>(p);
        r.get(v);
    } else {
        static_assert(V * sizeof(T) == 8);
        const uint2 h = *reinterpret_cast<const uint2 *>(p);
        Vec<T> r;
        float all[8];
        r.raw = make_uint4(h.x, h.y, 0, 0);
        r.get(all);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = all[i];
    }
}
template <typename T, int V>
__device__ __forceinline__ void store(T *p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = from_f32<T>(v[0]);
    } else if constexpr (V * sizeof(T) == 16) {
        Vec<T> r;
        r.set(v);
        *reinterpret_cast<uint4 *>(p) = r.raw;
    } else {
        float all[8] = {};
#pragma unroll
        for (int i = 0; i < V; ++i) all[i] = v[i];
        Vec<T> r;
        r.set(all);
        *reinterpret_cast<uint2 *>(p) = make_uint2(r.raw.x, r.raw.y);
    }
}

// The inputs in front of step t0 that it sees: rows t0 - W + 1 + i as h[i]; returns which ones lie behind the last flag (bit i).
template <typename T, int W, int V>
__device__ __forceinline__ int history(const ConvArgs &a, const T *x, const T *state, int e, int t0, float (&h)[W - 1][V]) {
    int seen = 0;
    bool cut = false;
#pragma unroll
    for (int i = W - 2; i >= 0; --i) {
        const int t = t0 - W + 1 + i;
        if (t >= 0 && a.done && a.done[(long long)t * a.Be + e]) cut = true;
#pragma unroll
        for (int v = 0; v < V; ++v) h[i][v] = 0.f;
        if (cut) continue;
        seen |= 1 << i;
        if (t >= 0) load(x + (long long)t * a.Be * a.ldx, h[i]);
        else if (state) load(state + (long long)(t + W - 1) * a.C, h[i]);
    }
    return seen;
}

template <int W, int V>
__device__ __forceinline__ void params(const ConvArgs &a, int c, float (&w)[W][V], float (&b)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        b[v] = a.bias ? a.bias[c + v] : 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) w[i][v] = a.weight[(long long)(c + v) * W + i];
    }
}

template <typename T, int W, int V>
__global__ void __launch_bounds__(256) conv_fwd_kernel(ConvArgs a) {
    grid_wait();
    const int cols = a.C / V;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, item = id / cols;
    const int c = (int)(id - item * cols) * V, tile = (int)(item / a.Be), e = (int)(item - (long long)tile * a.Be);
    if (tile >= a.tiles) return;
    const T *x = static_cast<const T *>(a.x) + e * a.ldx + c, *state = nullptr;
    T *y = static_cast<T *>(a.y) + e * a.ldy + c;
    const uint8_t *done = a.done ? a.done + e : nullptr;
    const long long sx = (long long)a.Be * a.ldx, sy = (long long)a.Be * a.ldy;
    if (a.state_in) state = static_cast<const T *>(a.state_in) + (long long)e * (W - 1) * a.C + c;
    float w[W][V], b[V], h[W - 1][V];
    params(a, c, w, b);
    const int t0 = tile * a.run, t1 = min(a.T, t0 + a.run);
    history<T, W, V>(a, x, state, e, t0, h);
    for (int t = t0; t < t1; t += 4) {
        float in[4][V];
        bool flag[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            flag[j] = false;
            if (t + j < t1) {
                load(x + (t + j) * sx, in[j]);
                flag[j] = done && done[(long long)(t + j) * a.Be];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (t + j >= t1) break;
            float o[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s = b[v];
#pragma unroll
                for (int i = 0; i < W - 1; ++i) s = fmaf(w[i][v], h[i][v], s);
                o[v] = activate(fmaf(w[W - 1][v], in[j][v], s), a.act);
#pragma unroll
                for (int i = 0; i < W - 2; ++i) h[i][v] = flag[j] ? 0.f : h[i + 1][v];
                h[W - 2][v] = flag[j] ? 0.f : in[j][v];
            }
            store(y + (t + j) * sy, o);
        }
    }
    // the first run writes the state that is left: it alone reads the one that came in, which may be the same
    if (tile == 0 && a.state_out) {
        history<T, W, V>(a, x, state, e, a.T, h);
        T *out = static_cast<T *>(a.state_out) + (long long)e * (W - 1) * a.C + c;
#pragma unroll
        for (int i = 0; i < W - 1; ++i) store(out + (long long)i * a.C, h[i]);
    }
}

// One step, the state in place.
template <typename T, int W, int V>
__global__ void __launch_bounds__(256) conv_step_kernel(ConvArgs a) {
    grid_wait();
    const int cols = a.C / V;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, e = id / cols;
    const int c = (int)(id - e * cols) * V;
    if (e >= a.Be) return;
    float w[W][V], b[V], h[W][V], o[V];
    T *state = static_cast<T *>(a.state_out) + e * (W - 1) * a.C + c;
    const bool start = a.done && a.done[e];
    load(static_cast<const T *>(a.x) + e * a.ldx + c, h[W - 1]);
#pragma unroll
    for (int i = 0; i < W - 1; ++i) load(state + (long long)i * a.C, h[i]);
    params(a, c, w, b);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float s = b[v];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (i < W - 1 && start) h[i][v] = 0.f;
            s = fmaf(w[i][v], h[i][v], s);
        }
        o[v] = activate(s, a.act);
    }
    store(static_cast<T *>(a.y) + e * a.ldy + c, o);
#pragma unroll
    for (int i = 0; i < W - 1; ++i) store(state + (long long)i * a.C, h[i + 1]);
}

// Gradients of a run: its own rows' sums are made again, those of the width - 1 steps behind it as well, whose gradients reach back.  Threads
// (p, l): l columns of V channels side by side, p runs; a thread takes every so many of them and keeps its shares of the gradients of weight
// and bias.
template <typename T, int W, int V>
__global__ void __launch_bounds__(256) conv_bwd_kernel(ConvArgs a, int lanes) {
    grid_wait();
    __shared__ float sum[256];
    const int l = threadIdx.x % lanes, p = threadIdx.x / lanes, rows = 256 / lanes, c = (blockIdx.x * lanes + l) * V;
    const bool on = c < a.C;
    const long long sx = (long long)a.Be * a.ldx, sy = (long long)a.Be * a.ldy;
    float w[W][V] = {}, b[V] = {}, dw[W][V] = {}, db[V] = {};
    if (on) params(a, c, w, b);
    const long long items = (long long)a.Be * a.tiles;
    for (long long item = (long long)blockIdx.y * rows + p; on && item < items; item += (long long)gridDim.y * rows) {
        const int tile = (int)(item / a.Be), e = (int)(item - (long long)tile * a.Be);
        const T *x = static_cast<const T *>(a.x) + e * a.ldx + c, *dy = static_cast<const T *>(a.dy) + e * a.ldy + c;
        T *dx = static_cast<T *>(a.dx) + e * a.ldx + c;
        const uint8_t *done = a.done ? a.done + e : nullptr;
        const long long states = (long long)e * (W - 1) * a.C + c;
        const T *state = a.state_in ? static_cast<const T *>(a.state_in) + states : nullptr;
        T *dstate = a.dstate_in ? static_cast<T *>(a.dstate_in) + states : nullptr;
        const int t0 = tile * a.run, t1 = min(a.T, t0 + a.run), end = min(a.T, t1 + W - 1);
        float h[W - 1][V], acc[W][V] = {};
        int seen = history<T, W, V>(a, x, state, e, t0, h) | 1 << (W - 1);
        const auto put = [&](int t, const float (&g)[V]) {  // the gradient of the input of step t is complete
            if (t >= t0 && t < t1) store(dx + t * sx, g);
            else if (t < 0 && t >= 1 - W && dstate) store(dstate + (long long)(t + W - 1) * a.C, g);
        };
        for (int t = t0; t < end; ++t) {
            float in[V], g[V];
            load(x + t * sx, in);
            load(dy + t * sy, g);
            const bool flag = done && done[(long long)t * a.Be];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float s = b[v];
#pragma unroll
                for (int i = 0; i < W - 1; ++i) s = fmaf(w[i][v], h[i][v], s);
                g[v] *= grad_act(fmaf(w[W - 1][v], in[v], s), a.act);
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i][v] = fmaf(w[i][v], seen >> i & 1 ? g[v] : 0.f, acc[i][v]);
                if (t < t1) {
#pragma unroll
                    for (int i = 0; i < W - 1; ++i) dw[i][v] = fmaf(g[v], h[i][v], dw[i][v]);
                    dw[W - 1][v] = fmaf(g[v], in[v], dw[W - 1][v]);
                    db[v] += g[v];
                }
#pragma unroll
                for (int i = 0; i < W - 2; ++i) h[i][v] = flag ? 0.f : h[i + 1][v];
                h[W - 2][v] = flag ? 0.f : in[v];
            }
            put(t - W + 1, acc[0]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int i = 0; i < W - 1; ++i) acc[i][v] = acc[i + 1][v];
                acc[W - 1][v] = 0.f;
            }
            seen = (flag ? 0 : seen >> 1) | 1 << (W - 1);
        }
        if (end == a.T) {  // what is left of the sequence, and reaches on into the state
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                if (a.dstate_out && seen >> i & 1) {
                    float s[V];
                    load(static_cast<const T *>(a.dstate_out) + states + (long long)i * a.C, s);
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[i][v] += s[v];
                }
                put(a.T - W + 1 + i, acc[i]);
            }
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.y * a.C * (W + 1);
#pragma unroll
    for (int i = 0; i <= W; ++i) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            __syncthreads();
            sum[threadIdx.x] = i < W ? dw[i < W ? i : 0][v] : db[v];
            __syncthreads();
            if (p == 0 && on) {
                float s = 0.f;
                for (int k = 0; k < rows; ++k) s += sum[k * lanes + l];
                part[i < W ? (size_t)(c + v) * W + i : (size_t)a.C * W + c + v] = s;
            }
        }
    }
}

int check(const ppo_causal_conv_desc *d) {
    if (!d || d->T <= 0 || d->Be <= 0 || d->C <= 0) return PPO_ERR_INVALID_ARG;
    if (d->act < PPO_ACT_NONE || d->act > PPO_ACT_SILU || d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->ldx < d->C || d->ldy < d->C) return PPO_ERR_SHAPE;
    if (d->width < 2 || d->width > 8 || d->C > 0x0fffffff || (long long)d->T * d->Be > 0x7f000000ll) return PPO_ERR_UNSUPPORTED;
    return PPO_OK;
}
bool misaligned(std::initializer_list<const void *> ps, size_t a) {
    for (const void *p : ps)
        if (!ppo_aligned(p, a)) return true;
    return false;
}

ConvArgs args(const ppo_causal_conv_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *done) {
    ConvArgs a = {};
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.done = done;
    a.ldx = d->ldx;
    a.ldy = d->ldy;
    a.T = d->T;
    a.Be = d->Be;
    a.C = d->C;
    a.act = d->act;
    a.run = 32;
    a.tiles = ppo_cdiv(d->T, a.run);
    return a;
}

// Lanes, blocks of them along the channels, blocks along the runs; by sizes alone, so that the workspace and the order of sums go by them.
struct BwdPlan {
    int lanes, cols, blocks;
};
BwdPlan plan_bwd(const ppo_causal_conv_desc *d, int V) {
    BwdPlan p = {1, 0, 0};
    while (p.lanes < 32 && p.lanes * V < d->C) p.lanes *= 2;
    p.cols = ppo_cdiv(d->C, p.lanes * V);
    const long long items = (long long)d->Be * ppo_cdiv(d->T, 32);
    const long long all = (items + 256 / p.lanes - 1) / (256 / p.lanes), want = ppo_cdiv(4 * 148, p.cols);
    p.blocks = (int)(all < want ? all : want);
    return p;
}

// fn(T{}, width, vectors) for the type and width of the call.
template <typename F>
int with_width(const ppo_causal_conv_desc *d, F &&fn) {
    return with_elem(d->dtype, [&](auto t) -> int {
        switch (d->width) {
            case 2: return fn(t, std::integral_constant<int, 2>{});
            case 3: return fn(t, std::integral_constant<int, 3>{});
            case 4: return fn(t, std::integral_constant<int, 4>{});
            case 5: return fn(t, std::integral_constant<int, 5>{});
            case 6: return fn(t, std::integral_constant<int, 6>{});
            case 7: return fn(t, std::integral_constant<int, 7>{});
            default: return fn(t, std::integral_constant<int, 8>{});
        }
    });
}
// Whether V elements of every row are one aligned vector.
bool vectors(const ppo_causal_conv_desc *d, int V, std::initializer_list<const void *> ps) {
    return d->C % V == 0 && d->ldx % V == 0 && d->ldy % V == 0 && !misaligned(ps, V * elem_bytes(d->dtype));
}
constexpr int kV = 4;

}  // namespace

extern "C" size_t ppo_causal_conv_workspace_bytes(const ppo_causal_conv_desc *d) {
    if (check(d) != PPO_OK) return 0;
    const int one = plan_bwd(d, 1).blocks, many = plan_bwd(d, kV).blocks;
    return (size_t)(one > many ? one : many) * d->C * (d->width + 1) * sizeof(float);
}

extern "C" int ppo_causal_conv_fwd(const ppo_causal_conv_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *done,
                                   const void *state_in, void *y, void *state_out, void *stream) {
    PPO_TRY(check(d));
    if (!x || !weight || !y) return PPO_ERR_INVALID_ARG;
    if (misaligned({x, y, state_in, state_out}, elem_bytes(d->dtype)) || misaligned({weight, bias}, 4)) return PPO_ERR_ALIGN;
    ConvArgs a = args(d, x, weight, bias, done);
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    const bool vec = vectors(d, kV, {x, y, state_in, state_out});
    const long long threads = (long long)(vec ? d->C / kV : d->C) * d->Be * a.tiles;
    if (threads > 0x7fffffffll * 256) return PPO_ERR_UNSUPPORTED;
    return with_width(d, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        return ppo_launch(vec ? conv_fwd_kernel<T, W, kV> : conv_fwd_kernel<T, W, 1>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0,
                          static_cast<cudaStream_t>(stream), a);
    });
}

extern "C" int ppo_causal_conv_bwd(const ppo_causal_conv_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *done,
                                   const void *state_in, const void *dy, const void *dstate_out, void *dx, void *dstate_in, float *dweight,
                                   float *dbias, int accumulate, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    if (!x || !weight || !dy || !dx || !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < ppo_causal_conv_workspace_bytes(d)) return PPO_ERR_SHAPE;
    if (misaligned({x, dy, dx, state_in, dstate_out, dstate_in}, elem_bytes(d->dtype)) || misaligned({weight, bias, dweight, dbias}, 4) ||
        misaligned({workspace}, 32))
        return PPO_ERR_ALIGN;
    ConvArgs a = args(d, x, weight, bias, done);
    a.state_in = state_in;
    a.dy = dy;
    a.dstate_out = dstate_out;
    a.dx = dx;
    a.dstate_in = dstate_in;
    const bool params = dweight || dbias, vec = vectors(d, kV, {x, dy, dx, state_in, dstate_out, dstate_in});
    a.part = params ? static_cast<float *>(workspace) : nullptr;
    const BwdPlan p = plan_bwd(d, vec ? kV : 1);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    PPO_TRY(with_width(d, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        return ppo_launch(vec ? conv_bwd_kernel<T, W, kV> : conv_bwd_kernel<T, W, 1>, dim3(p.cols, p.blocks), dim3(256), 0, st, a, p.lanes);
    }));
    return params ? ppo_param_sum(a.part, p.blocks, {{dweight, dbias, nullptr}, {d->C * d->width, d->C, 0}}, accumulate, st) : PPO_OK;
}

extern "C" int ppo_causal_conv_step(const ppo_causal_conv_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *start,
                                    void *state, void *y, void *stream) {
    PPO_TRY(check(d));
    if (d->T != 1) return PPO_ERR_SHAPE;
    if (!x || !weight || !state || !y) return PPO_ERR_INVALID_ARG;
    if (misaligned({x, y, state}, elem_bytes(d->dtype)) || misaligned({weight, bias}, 4)) return PPO_ERR_ALIGN;
    ConvArgs a = args(d, x, weight, bias, start);
    a.y = y;
    a.state_out = state;
    const bool vec = vectors(d, kV, {x, y, state});
    const long long threads = (long long)(vec ? d->C / kV : d->C) * d->Be;
    if (threads > 0x7fffffffll * 256) return PPO_ERR_UNSUPPORTED;
    return with_width(d, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        return ppo_launch(vec ? conv_step_kernel<T, W, kV> : conv_step_kernel<T, W, 1>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0,
                          static_cast<cudaStream_t>(stream), a);
    });
}
