// Causal convolution of each channel along the steps of an env, with an activation, and its gradients.
//
// A thread takes V neighbouring channels over a run of steps of one env: every input is read once (but for the width - 1 in front of a run) and
// every output written once; the last width - 1 inputs stay in registers, found by their place in a ring that is known when this is compiled.
// A thread copies its own rows ahead into shared memory, a batch of rows at a time, and waits for nobody else.  Arithmetic on two
// channels in one instruction, sums in 32 bits.  8192 steps of 4096 bf16 channels with SiLU: 35 us, 3.8 TB/s, 47 % of the rate of exponentials and
// reciprocals (two an element); 16 warps an SM, as many as 122 registers leave.  Gradients of 16 steps of 256 envs of 2048: 31 us, 43 % of
// the issue slots (64 bytes a thread, the sums that the ends of runs choose from, lie in local memory); 512 decisions of 4096: 12.4.  Single elements, where
// 16 bytes do not fit the rows: 95 us for the first of these with 4092 channels, 84 for the gradients with 2046.
#include "approx.cuh"
#include "elem.cuh"
#include "pair32.cuh"
#include "param_sum.cuh"

namespace {

constexpr int kThreads = 128;

struct ConvArgs {
    const void *x, *state_in, *dy, *dstate_out;
    void *y, *state_out, *dx, *dstate_in;
    const float *weight, *bias;
    const uint8_t *done;
    float *part;  // shares of the gradients of weight and bias, [parts][C * width + C]
    long long ldx, ldy, sx, sy;  // from row to row, and from step to step
    int T, Be, C, act, run, tiles;
};

// V elements, aligned to all of them, as they lie in memory; V / 2 pairs of them in 32 bits (one, with a second channel of zeros, where V is 1).
template <typename T, int V>
struct Raw {
    static constexpr int BYTES = V * sizeof(T), PAIRS = (V + 1) / 2;
    static_assert(V == 1 || BYTES == 8 || BYTES == 16);
    using Word = std::conditional_t<V == 1, T, std::conditional_t<BYTES == 8, uint2, uint4>>;
    Word w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const Word *>(p); }
    __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<Word *>(p) = w; }
    __device__ __forceinline__ void get(pair32 (&v)[PAIRS]) const {
        if constexpr (V == 1) {
            v[0] = pair_of(to_f32(w), 0.f);
        } else {
            Vec<T> all;
            float f[Vec<T>::N];
            if constexpr (BYTES == 8) all.raw = make_uint4(w.x, w.y, 0, 0);
            else all.raw = w;
            all.get(f);
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) v[i] = pair_of(f[2 * i], f[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void set(const pair32 (&v)[PAIRS]) {
        if constexpr (V == 1) {
            w = from_f32<T>(parts(v[0]).x);
        } else {
            Vec<T> all;
            float f[Vec<T>::N] = {};
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                const float2 p = parts(v[i]);
                f[2 * i] = p.x, f[2 * i + 1] = p.y;
            }
            all.set(f);
            if constexpr (BYTES == 8) w = make_uint2(all.raw.x, all.raw.y);
            else w = all.raw;
        }
    }
};

// A thread's places in a ring of shared memory: S rows of V elements.
template <typename T, int V, int S>
struct Ring {
    using Word = typename Raw<T, V>::Word;
    Word (*at)[kThreads];
    __device__ __forceinline__ void copy(int slot, const T *from) const {
        if constexpr (V == 1) {
            at[slot][threadIdx.x] = *from;
        } else {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(&at[slot][threadIdx.x]);
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(Raw<T, V>::BYTES) : "memory");
        }
    }
    __device__ __forceinline__ void get(int slot, Raw<T, V> &r) const { r.w = at[slot][threadIdx.x]; }
};
__device__ __forceinline__ void batch_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All batches but the N youngest have arrived.
template <int N>
__device__ __forceinline__ void batch_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// act(z), in place
template <int P>
__device__ __forceinline__ void activate(pair32 (&z)[P], int act) {
    if (act == PPO_ACT_SILU) {
#pragma unroll
        for (int p = 0; p < P; ++p) z[p] = mul2(z[p], sigmoid_pair(z[p]));
    } else if (act == PPO_ACT_RELU) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const float2 f = parts(z[p]);
            z[p] = pair_of(f.x < 0.f ? 0.f : f.x, f.y < 0.f ? 0.f : f.y);  // a NaN stays
        }
    }
}
// g act'(z), in place; s (1 + z (1 - s)) with s = sigmoid(z) for SiLU
template <int P>
__device__ __forceinline__ void through_act(pair32 (&g)[P], const pair32 (&z)[P], int act) {
    if (act == PPO_ACT_SILU) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const pair32 one = pair_of(1.f, 1.f), s = sigmoid_pair(z[p]), rest = fma2(s, pair_of(-1.f, -1.f), one);
            g[p] = mul2(g[p], mul2(s, fma2(z[p], rest, one)));
        }
    } else if (act == PPO_ACT_RELU) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const float2 f = parts(z[p]), v = parts(g[p]);
            g[p] = pair_of(f.x > 0.f ? v.x : 0.f, f.y > 0.f ? v.y : 0.f);
        }
    }
}

// The inputs in front of step t0 that it sees: rows t0 - W + 1 + i as h[i]; returns which ones lie behind the last flag (bit i).
template <typename T, int W, int V, int P>
__device__ __forceinline__ int history(const ConvArgs &a, const T *x, const T *state, int e, int t0, pair32 (&h)[W - 1][P]) {
    int seen = 0;
    bool cut = false;
#pragma unroll
    for (int i = W - 2; i >= 0; --i) {
        const int t = t0 - W + 1 + i;
        if (t >= 0 && a.done && a.done[(long long)t * a.Be + e]) cut = true;
#pragma unroll
        for (int p = 0; p < P; ++p) h[i][p] = 0;
        if (cut) continue;
        seen |= 1 << i;
        Raw<T, V> r;
        if (t >= 0) r.load(x + (long long)t * a.Be * a.ldx);
        else if (state) r.load(state + (long long)(t + W - 1) * a.C);
        else continue;
        r.get(h[i]);
    }
    return seen;
}

template <int W, int V, int P>
__device__ __forceinline__ void params(const ConvArgs &a, int c, pair32 (&w)[W][P], pair32 (&b)[P]) {
    float f[2 * P * W] = {}, g[2 * P] = {};
    const float *from = a.weight + (long long)c * W;
    if (V % 4 == 0 && (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < V * W / 4; ++i) {
            const float4 v = reinterpret_cast<const float4 *>(from)[i];
            f[4 * i] = v.x, f[4 * i + 1] = v.y, f[4 * i + 2] = v.z, f[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V * W; ++i) f[i] = from[i];
    }
    if (V % 4 == 0 && a.bias && (reinterpret_cast<uintptr_t>(a.bias) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float4 v = reinterpret_cast<const float4 *>(a.bias + c)[i];
            g[4 * i] = v.x, g[4 * i + 1] = v.y, g[4 * i + 2] = v.z, g[4 * i + 3] = v.w;
        }
    } else if (a.bias) {
#pragma unroll
        for (int v = 0; v < V; ++v) g[v] = a.bias[c + v];
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        b[p] = pair_of(g[2 * p], g[2 * p + 1]);
#pragma unroll
        for (int i = 0; i < W; ++i) w[i][p] = pair_of(f[2 * p * W + i], f[(2 * p + 1) * W + i]);
    }
}

template <typename T, int W, int V>
__global__ void __launch_bounds__(kThreads) conv_fwd_kernel(ConvArgs a) {
    grid_wait();
    // batches of BATCH rows, AHEAD of them on their way; a multiple of W, so that which input lies how far back is known when this is compiled
    constexpr int P = Raw<T, V>::PAIRS, BATCH = W == 2 ? 4 : W, AHEAD = W <= 6 ? 3 : 2, S = BATCH * (AHEAD + 1);
    __shared__ typename Raw<T, V>::Word rows[S][kThreads];
    const Ring<T, V, S> ring = {rows};
    const int cols = a.C / V;
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x, item = id / cols;
    const int c = (int)(id - item * cols) * V, tile = (int)(item / a.Be), e = (int)(item - (long long)tile * a.Be);
    if (tile >= a.tiles) return;
    const T *x = static_cast<const T *>(a.x) + e * a.ldx + c, *state = nullptr;
    const uint8_t *done = a.done ? a.done + e : nullptr;
    const long long &sx = a.sx, &sy = a.sy;
    if (a.state_in) state = static_cast<const T *>(a.state_in) + (long long)e * (W - 1) * a.C + c;
    const int t0 = tile * a.run, t1 = min(a.T, t0 + a.run);
    const T *ahead = x + t0 * sx;
    T *out = static_cast<T *>(a.y) + e * a.ldy + c + t0 * sy;
    int left = t1 - t0, to = 0;  // rows that are not fetched yet, and where in the ring the next batch goes
    const auto fetch = [&] {
#pragma unroll
        for (int j = 0; j < BATCH; ++j)
            if (j < left) ring.copy(to + j, ahead + j * sx);
        batch_end();
        left -= BATCH;
        ahead += BATCH * sx;
        to = to + BATCH == S ? 0 : to + BATCH;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch();
    pair32 w[W][P], b[P], h[W][P];  // h[t % W]: the input of step t0 + t
    params<W, V>(a, c, w, b);
    {
        pair32 f[W - 1][P];
        history<T, W, V>(a, x, state, e, t0, f);
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
#pragma unroll
            for (int p = 0; p < P; ++p) h[i + 1][p] = f[i][p];
    }
    int from = 0;
    for (int t = t0; t < t1; t += BATCH) {
        fetch();
        bool flag[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) flag[j] = done && t + j < t1 && done[(long long)(t + j) * a.Be];
        batch_wait<AHEAD>();
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (t + j >= t1) break;
            Raw<T, V> r;
            pair32 o[P];
            ring.get(from + j, r);
            r.get(h[j % W]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                o[p] = b[p];
#pragma unroll
                for (int i = 0; i < W; ++i) o[p] = fma2(w[i][p], h[(j + 1 + i) % W][p], o[p]);
            }
            if (flag[j]) {
#pragma unroll
                for (int i = 0; i < W; ++i)
#pragma unroll
                    for (int p = 0; p < P; ++p) h[i][p] = 0;
            }
            activate(o, a.act);
            r.set(o);
            r.store(out);
            out += sy;
        }
        from = from + BATCH == S ? 0 : from + BATCH;
    }
    // the first run writes the state that is left: it alone reads the one that came in, which may be the same
    if (tile == 0 && a.state_out) {
        pair32 f[W - 1][P];
        history<T, W, V>(a, x, state, e, a.T, f);
        T *to = static_cast<T *>(a.state_out) + (long long)e * (W - 1) * a.C + c;
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            Raw<T, V> r;
            r.set(f[i]);
            r.store(to + (long long)i * a.C);
        }
    }
}

// One step of `envs` envs, the state in place.
template <typename T, int W, int V>
__global__ void __launch_bounds__(kThreads) conv_step_kernel(ConvArgs a, int envs) {
    grid_wait();
    constexpr int P = Raw<T, V>::PAIRS;
    const int cols = a.C / V;
    const long long id = (long long)blockIdx.x * kThreads + threadIdx.x, item = id / cols;
    const int c = (int)(id - item * cols) * V;
    if (item * envs >= a.Be) return;
    const int e0 = (int)item * envs, e1 = min(a.Be, e0 + envs);
    Raw<T, V> r[2][W];
    bool start[2];
    T *const states = static_cast<T *>(a.state_out) + c;
    const long long each = (long long)(W - 1) * a.C;
    const auto read = [&](int e) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (e + k >= e1) break;
            start[k] = a.done && a.done[e + k];
            r[k][W - 1].load(static_cast<const T *>(a.x) + (e + k) * a.ldx + c);
#pragma unroll
            for (int i = 0; i < W - 1; ++i) r[k][i].load(states + (e + k) * each + (long long)i * a.C);
        }
    };
    read(e0);
    pair32 w[W][P], b[P];
    params<W, V>(a, c, w, b);
    for (int e = e0; e < e1; e += 2) {
        if (e > e0) read(e);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (e + k >= e1) break;
            pair32 s[P], v[P];
#pragma unroll
            for (int p = 0; p < P; ++p) s[p] = b[p];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (i < W - 1 && start[k]) r[k][i].w = typename Raw<T, V>::Word{};
                r[k][i].get(v);
#pragma unroll
                for (int p = 0; p < P; ++p) s[p] = fma2(w[i][p], v[p], s[p]);
                if (i > 0) r[k][i].store(states + (e + k) * each + (long long)(i - 1) * a.C);
            }
            activate(s, a.act);
            r[k][0].set(s);
            r[k][0].store(static_cast<T *>(a.y) + (e + k) * a.ldy + c);
        }
    }
}

// Gradients of a run: its own rows' sums are made again, those of the width - 1 steps behind it as well, whose gradients reach back.  Threads
// (p, l): l columns of V channels side by side, p runs; a thread takes every so many of them and keeps its shares of the gradients of weight
// and bias.
template <typename T, int W, int V>
__global__ void __launch_bounds__(kThreads, W <= 4 ? 4 : 2) conv_bwd_kernel(ConvArgs a, int lanes) {
    grid_wait();
    constexpr int P = Raw<T, V>::PAIRS, BATCH = W == 2 ? 4 : W, AHEAD = W <= 4 ? 2 : 1, S = BATCH * (AHEAD + 1), ALL = (1 << W) - 1;
    using Word = typename Raw<T, V>::Word;
    constexpr int SUMS = (W + 1) * V;
    // the rings of x and dy; behind the last run, the sums of all threads
    __shared__ alignas(16) char shared[2 * S * sizeof(Word) > SUMS * sizeof(float) ? 2 * S * sizeof(Word) * kThreads : SUMS * sizeof(float) * kThreads];
    const Ring<T, V, S> xs = {reinterpret_cast<Word(*)[kThreads]>(shared)}, gs = {xs.at + S};
    float(*const sums)[kThreads] = reinterpret_cast<float(*)[kThreads]>(shared);
    const int l = threadIdx.x % lanes, p0 = threadIdx.x / lanes, rows = kThreads / lanes, c = (blockIdx.x * lanes + l) * V;
    const bool on = c < a.C;
    const long long &sx = a.sx, &sy = a.sy;
    pair32 w[W][P] = {}, b[P] = {}, dw[W][P] = {}, db[P] = {};
    if (on) params<W, V>(a, c, w, b);
    const long long items = (long long)a.Be * a.tiles;
    for (long long item = (long long)blockIdx.y * rows + p0; on && item < items; item += (long long)gridDim.y * rows) {
        const int tile = (int)(item / a.Be), e = (int)(item - (long long)tile * a.Be);
        const T *x = static_cast<const T *>(a.x) + e * a.ldx + c;
        const uint8_t *done = a.done ? a.done + e : nullptr;
        const long long states = (long long)e * (W - 1) * a.C + c;
        const T *state = a.state_in ? static_cast<const T *>(a.state_in) + states : nullptr;
        T *dstate = a.dstate_in ? static_cast<T *>(a.dstate_in) + states : nullptr;
        const int t0 = tile * a.run, t1 = min(a.T, t0 + a.run), end = min(a.T, t1 + W - 1);
        const T *ahead = x + t0 * sx, *gahead = static_cast<const T *>(a.dy) + e * a.ldy + c + t0 * sy;
        int left = end - t0, to = 0;
        const auto fetch = [&] {
#pragma unroll
            for (int j = 0; j < BATCH; ++j)
                if (j < left) {
                    xs.copy(to + j, ahead + j * sx);
                    gs.copy(to + j, gahead + j * sy);
                }
            batch_end();
            left -= BATCH;
            ahead += BATCH * sx;
            gahead += BATCH * sy;
            to = to + BATCH == S ? 0 : to + BATCH;
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch();
        // h[t % W]: the input of step t0 + t, acc[t % W]: its gradient; bit i of seen: whether step t still sees the input of step t - W + 1 + i
        pair32 h[W][P], acc[W][P] = {};
        int seen;
        {
            pair32 f[W - 1][P];
            seen = history<T, W, V>(a, x, state, e, t0, f) | 1 << (W - 1);
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) h[i + 1][p] = f[i][p];
        }
        T *dx = static_cast<T *>(a.dx) + e * a.ldx + c + (t0 - W + 1) * sx;  // of the step whose gradient is complete next
        const auto put = [&](int t, const pair32 (&g)[P]) {
            Raw<T, V> r;
            r.set(g);
            if (t >= t0) {
                if (t < t1) r.store(dx);
            } else if (t < 0 && t >= 1 - W && dstate) {
                r.store(dstate + (long long)(t + W - 1) * a.C);
            }
            dx += sx;
        };
        int from = 0;
        for (int t = t0; t < end; t += BATCH) {
            fetch();
            bool flag[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) flag[j] = done && t + j < end && done[(long long)(t + j) * a.Be];
            batch_wait<AHEAD>();
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                if (t + j >= end) break;
                pair32 g[P], z[P];
                Raw<T, V> r;
                xs.get(from + j, r);
                r.get(h[j % W]);
                gs.get(from + j, r);
                r.get(g);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    z[p] = b[p];
#pragma unroll
                    for (int i = 0; i < W; ++i) z[p] = fma2(w[i][p], h[(j + 1 + i) % W][p], z[p]);
                }
                through_act(g, z, a.act);
                if (seen == ALL) {
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int p = 0; p < P; ++p) acc[(j + 1 + i) % W][p] = fma2(w[i][p], g[p], acc[(j + 1 + i) % W][p]);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        if (seen >> i & 1) {
#pragma unroll
                            for (int p = 0; p < P; ++p) acc[(j + 1 + i) % W][p] = fma2(w[i][p], g[p], acc[(j + 1 + i) % W][p]);
                        }
                }
                if (t + j < t1) {
#pragma unroll
                    for (int p = 0; p < P; ++p) {
#pragma unroll
                        for (int i = 0; i < W; ++i) dw[i][p] = fma2(g[p], h[(j + 1 + i) % W][p], dw[i][p]);
                        db[p] = add2(db[p], g[p]);
                    }
                }
                put(t + j - W + 1, acc[(j + 1) % W]);
#pragma unroll
                for (int p = 0; p < P; ++p) acc[(j + 1) % W][p] = 0;
                seen = seen >> 1 | 1 << (W - 1);
                if (flag[j]) {
                    seen = 1 << (W - 1);
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int p = 0; p < P; ++p) h[i][p] = 0;
                }
            }
            from = from + BATCH == S ? 0 : from + BATCH;
        }
        batch_wait<0>();
        // What is left at the end of the sequence reaches on into the state.  Behind the last step, of which there were end - t0, the gradient of the
        // input i steps from the oldest one is acc[(end - t0 + i + 1) % W].
        if (end == a.T) {
            const int turn = (end - t0) % W;
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                pair32 s[P] = {};
                if (a.dstate_out && seen >> i & 1) {
                    Raw<T, V> r;
                    r.load(static_cast<const T *>(a.dstate_out) + states + (long long)i * a.C);
                    r.get(s);
                }
#pragma unroll
                for (int k = 0; k < W; ++k)
                    if ((turn + i + 1) % W == k) {
#pragma unroll
                        for (int p = 0; p < P; ++p) s[p] = add2(acc[k][p], s[p]);
                    }
                put(a.T - W + 1 + i, s);
            }
        }
    }
    if (!a.part) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SUMS; ++i) {
        const float2 f = parts(i < W * V ? dw[i < W * V ? i / V : 0][i % V / 2] : db[i % V / 2]);
        sums[i][threadIdx.x] = i % V % 2 ? f.y : f.x;
    }
    __syncthreads();
    float *part = a.part + (size_t)blockIdx.y * a.C * (W + 1);
    for (int o = threadIdx.x; o < SUMS * lanes; o += kThreads) {
        const int i = o / lanes, at = o % lanes, to = (blockIdx.x * lanes + at) * V + i % V;
        if (to >= a.C) continue;
        float s = 0.f;
        for (int k = 0; k < rows; ++k) s += sums[i][k * lanes + at];
        part[i < W * V ? (size_t)to * W + i / V : (size_t)a.C * W + to] = s;
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

constexpr int kRun = 32;  // steps of a run

ConvArgs args(const ppo_causal_conv_desc *d, const void *x, const float *weight, const float *bias, const uint8_t *done) {
    ConvArgs a = {};
    a.x = x;
    a.weight = weight;
    a.bias = bias;
    a.done = done;
    a.ldx = d->ldx;
    a.ldy = d->ldy;
    a.sx = d->Be * d->ldx;
    a.sy = d->Be * d->ldy;
    a.T = d->T;
    a.Be = d->Be;
    a.C = d->C;
    a.act = d->act;
    a.run = kRun;
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
    const long long items = (long long)d->Be * ppo_cdiv(d->T, kRun);
    const long long all = (items + kThreads / p.lanes - 1) / (kThreads / p.lanes), want = p.cols < 4 * 148 ? 4 * 148 / p.cols : 1;  // one round of four blocks an SM
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
// Channels of a thread: 16 bytes of them, but 8 bytes in the gradients, whose shares need the registers.
int bwd_v(const ppo_causal_conv_desc *d) { return 8 / (int)elem_bytes(d->dtype); }
// fn(T{}, width, V)
template <typename F>
int with_columns(const ppo_causal_conv_desc *d, bool vec, F &&fn) {
    return with_width(d, [&](auto t, auto w) -> int {
        constexpr int V = 16 / (int)sizeof(t);
        return vec ? fn(t, w, std::integral_constant<int, V>{}) : fn(t, w, std::integral_constant<int, 1>{});
    });
}

}  // namespace

extern "C" size_t ppo_causal_conv_workspace_bytes(const ppo_causal_conv_desc *d) {
    if (check(d) != PPO_OK) return 0;
    const int one = plan_bwd(d, 1).blocks, many = plan_bwd(d, bwd_v(d)).blocks;
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
    const int V = 16 / (int)elem_bytes(d->dtype);
    const bool vec = vectors(d, V, {x, y, state_in, state_out});
    const long long blocks = ((long long)(vec ? d->C / V : d->C) * d->Be * a.tiles + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffll) return PPO_ERR_UNSUPPORTED;
    return with_columns(d, vec, [&](auto t, auto w, auto v) -> int {
        return ppo_launch(conv_fwd_kernel<decltype(t), decltype(w)::value, decltype(v)::value>, dim3((unsigned)blocks), dim3(kThreads), 0,
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
    const bool params = dweight || dbias, vec = vectors(d, bwd_v(d), {x, dy, dx, state_in, dstate_out, dstate_in});
    a.part = params ? static_cast<float *>(workspace) : nullptr;
    const BwdPlan p = plan_bwd(d, vec ? bwd_v(d) : 1);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    PPO_TRY(with_width(d, [&](auto t, auto w) -> int {
        using T = decltype(t);
        constexpr int W = decltype(w)::value;
        return ppo_launch(vec ? conv_bwd_kernel<T, W, 8 / (int)sizeof(T)> : conv_bwd_kernel<T, W, 1>, dim3(p.cols, p.blocks), dim3(kThreads), 0, st, a, p.lanes);
    }));
    return params ? ppo_param_sum(a.part, p.blocks, {{dweight, dbias, nullptr}, {(long long)d->C * d->width, d->C, 0}}, accumulate, st) : PPO_OK;
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
    const int V = 16 / (int)elem_bytes(d->dtype);
    const bool vec = vectors(d, V, {x, y, state});
    const long long cols = vec ? d->C / V : d->C, most = cols * d->Be / (148 * 256);  // envs of a thread: as many as leave every SM 256 threads
    const int envs = most < 2 ? 1 : most > 8 ? 8 : (int)most / 2 * 2;
    const long long blocks = (cols * ppo_cdiv(d->Be, envs) + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffll) return PPO_ERR_UNSUPPORTED;
    return with_columns(d, vec, [&](auto t, auto w, auto v) -> int {
        return ppo_launch(conv_step_kernel<decltype(t), decltype(w)::value, decltype(v)::value>, dim3((unsigned)blocks), dim3(kThreads), 0,
                          static_cast<cudaStream_t>(stream), a, envs);
    });
}
