// Norms of queries and keys for each head with the rotation by their positions, and the gradients.
//
// Angles in 64 bits down to the fraction of a turn, which fits 32; the rest in 32 bits; what is stored is rounded once.  Everything is read and
// written once.  A warp takes the heads of a row side by side, a few lanes each, two vectors of four elements a lane such that a lane has both
// elements of every pair it turns; the row's cosines and sines are made once for all its heads, d / 64 of them a lane.  16384 rows of 20 heads of
// 128 bf16: 40 us, 4.2 TB/s, 69 % of the issue slots; gradients of 4096 rows of 32 heads of 64: 20 us with the launch that sums the shares, bound
// by the chain from a row's position to its turns and sums.  Vectors of eight elements (half as many warps an SM): 44 and 27.
#include <cfloat>

#include "elem.cuh"
#include "pair32.cuh"
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
    float eps, inv_d;
};

constexpr double kTurn = 0.15915494309189535;  // of a radian
// cos and sin of the angle pos * f, f in turns.
__device__ __forceinline__ float2 turn(int pos, double f) {
    const double t = (double)pos * f;
    float2 r;
    sincospif((float)(2. * (t - rint(t))), &r.y, &r.x);
    return r;
}
// 1 / sqrt(sum / d + eps): the hardware's approximation and a step of Newton's method, which leaves a unit of the last place.  SMALL: of a mean below the
// normal numbers as well, which an eps below them allows (41.0 us where the larger case above takes 40.4, so not for every eps).
template <bool SMALL>
__device__ __forceinline__ float root(const QkArgs &a, float sum) {
    const float m = fmaf(sum, a.inv_d, a.eps);
    float r;
    if (SMALL) asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(m));
    else asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(m));
    const float h = 0.5f * m * r;
    return m > 3e38f ? r : fmaf(r, fmaf(-h, r, 0.5f), r);  // an infinite sum makes zeros
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

// ---- any size and alignment: a warp per head, element by element (the larger case above with heads of 100: 342 us, the gradients 108) ----

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
        const T *x = key ? static_cast<const T *>(a.k) + row * a.ldk + (long long)(h - a.heads) * a.d : static_cast<const T *>(a.q) + row * a.ldq + (long long)h * a.d;
        T *y = key ? static_cast<T *>(a.ko) + row * a.ldko + (long long)(h - a.heads) * a.d : static_cast<T *>(a.qo) + row * a.ldqo + (long long)h * a.d;
        const float *gamma = key ? a.gamma_k : a.gamma_q;
        float s = 0.f;
        for (int i = lane; i < a.d; i += 32) {
            n[i] = to_f32(x[i]);
            s = fmaf(n[i], n[i], s);
        }
        const float r = root<true>(a, warp_sum(s));
        for (int i = lane; i < a.d; i += 32) n[i] *= r * (gamma ? gamma[i] : 1.f);
        __syncwarp();
        for (int i = lane; i < a.d; i += 32) {
            const Place p = place(a, i);
            float v = n[i];
            if (p.pair >= 0) {
                const float2 t = turn(a.pos[row], a.freq[p.pair] * kTurn);
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
        const T *x = key ? static_cast<const T *>(a.k) + row * a.ldk + (long long)(h - a.heads) * a.d : static_cast<const T *>(a.q) + row * a.ldq + (long long)h * a.d;
        const T *dy = key ? static_cast<const T *>(a.dko) + row * a.ldko + (long long)(h - a.heads) * a.d : static_cast<const T *>(a.dqo) + row * a.ldqo + (long long)h * a.d;
        T *dx = key ? static_cast<T *>(a.dk) + row * a.ldk + (long long)(h - a.heads) * a.d : static_cast<T *>(a.dq) + row * a.ldq + (long long)h * a.d;
        const float *gamma = key ? a.gamma_k : a.gamma_q;
        float v[kMaxD / 32], s = 0.f;
#pragma unroll
        for (int j = 0; j < kMaxD / 32; ++j) {
            const int i = lane + 32 * j;
            v[j] = i < a.d ? to_f32(x[i]) : 0.f;
            if (i < a.d) n[i] = to_f32(dy[i]);
            s = fmaf(v[j], v[j], s);
        }
        const float r = root<true>(a, warp_sum(s));
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
                const float2 t = turn(a.pos[row], a.freq[p.pair] * kTurn);
                g[j] = p.second ? fmaf(-n[p.other], t.y, g[j] * t.x) : fmaf(n[p.other], t.y, g[j] * t.x);
            }
            v[j] *= r;
            sum[key][j] = fmaf(g[j], v[j], sum[key][j]);
            g[j] *= gamma ? gamma[i] : 1.f;
            dot = fmaf(g[j], v[j], dot);
        }
        dot = warp_sum(dot) * a.inv_d;
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

// ---- rows of aligned vectors ----

// Four elements: what a lane has of a head is two times four.
template <typename T>
struct Four {
    using Word = std::conditional_t<sizeof(T) == 4, uint4, uint2>;
};

// How the warps go about it: lanes of a head (a power of two, of which `slots` hold something), the parts that a row's heads are dealt to, heads
// of a part.
struct Lanes {
    int lanes, slots, parts, heads;
    int warps;  // of a block, for the queries (gradients, where a warp has either queries or keys)
};

// The row's turns, and where a lane's two vectors stand in a head.  ALL: every pair of every head is turned.
template <typename T, bool INTERLEAVED, bool ALL>
struct Turns {
    static constexpr int V = 4, P = V / 2;
    int first, second, own;  // own: how many of the lane's four pairs of neighbours are turned; the others have nothing to do with one another
    bool on;
    pair32 c[P], s[P], n[P];  // of two pairs each: cosines, sines, and these negative
    double f[kMaxD / 64];     // turns a position of the pairs that a lane makes

    __device__ __forceinline__ Turns(const QkArgs &a, const Lanes &k) {
        const int slot = threadIdx.x % k.lanes, turned = a.pairs / V;  // slots whose vectors are turned with one another
        on = slot < k.slots;
#pragma unroll
        for (int i = 0; i < kMaxD / 64; ++i) {
            const int p = threadIdx.x % 32 + 32 * i;
            f[i] = p < a.pairs ? a.freq[p] * kTurn : 0.;
        }
        if (INTERLEAVED) {
            first = 2 * V * slot;
            second = first + V;
        } else if (slot < turned) {
            first = V * slot;
            second = a.pairs + first;
        } else {
            first = 2 * a.pairs + 2 * V * (slot - turned);
            second = first + V;
        }
        own = INTERLEAVED && on ? max(0, min(V, a.pairs - first / 2)) : 0;
    }
    // table: of the warp; made by all its lanes
    __device__ __forceinline__ void row(const QkArgs &a, long long row, float2 *table) {
        __syncwarp();
        if (a.pairs > 0) {
            const int pos = a.pos[row];
#pragma unroll
            for (int i = 0; i < kMaxD / 64; ++i)
                if ((int)threadIdx.x % 32 + 32 * i < a.pairs) table[threadIdx.x % 32 + 32 * i] = turn(pos, f[i]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float2 t = make_float2(1.f, 0.f), u = t;
            const int p = (INTERLEAVED ? first / 2 : first) + 2 * i;
            if (on && p < a.pairs) t = table[p];
            if (on && p + 1 < a.pairs) u = table[p + 1];
            c[i] = pair_of(t.x, u.x), s[i] = pair_of(t.y, u.y), n[i] = pair_of(-t.y, -u.y);
        }
    }
    static __device__ __forceinline__ pair32 swap(pair32 p) {
        const float2 f = parts(p);
        return pair_of(f.y, f.x);
    }
    // a c + b where it is turned, else a
    static __device__ __forceinline__ void add_if(bool turned, pair32 &a, pair32 c, pair32 b) {
        if (ALL) a = fma2(a, c, b);
        else asm("{\n.reg .pred p;\nsetp.ne.s32 p, %3, 0;\n@p fma.rn.f32x2 %0, %0, %1, %2;\n}" : "+l"(a) : "l"(c), "l"(b), "r"((int)turned));
    }
    // x: the pairs of neighbours of both vectors; BACK: by the opposite angle.  Pairs that stay are left out by a predicate or by a branch, whichever
    // takes less (half of each head turned: 40.4 us where neighbours are turned with one another, by a branch 41.4; 41.6 by halves, 43.1 by a
    // predicate; 38.9 and 40.9 without either).
    template <bool BACK>
    __device__ __forceinline__ void apply(const QkArgs &k, pair32 (&x)[V]) const {
        if constexpr (INTERLEAVED) {
            if (BACK && !ALL && own == 0) return;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 ct = parts(c[i / 2]), st = parts(BACK ? n[i / 2] : s[i / 2]), nt = parts(BACK ? s[i / 2] : n[i / 2]);
                add_if(i < own, x[i], i % 2 ? pair_of(ct.y, ct.y) : pair_of(ct.x, ct.x), mul2(swap(x[i]), i % 2 ? pair_of(nt.y, st.y) : pair_of(nt.x, st.x)));
            }
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const pair32 b = mul2(x[P + i], BACK ? s[i] : n[i]), a = mul2(x[i], BACK ? n[i] : s[i]);
                if (ALL || first < k.pairs) x[i] = fma2(x[i], c[i], b), x[P + i] = fma2(x[P + i], c[i], a);
            }
        }
    }
};

template <typename T>
__device__ __forceinline__ void pairs_of(const typename Four<T>::Word &raw, pair32 *p) {
    Vec<T> v;
    float f[Vec<T>::N];
    if constexpr (sizeof(T) == 4) v.raw = raw;
    else v.raw = make_uint4(raw.x, raw.y, 0, 0);
    v.get(f);
    p[0] = pair_of(f[0], f[1]), p[1] = pair_of(f[2], f[3]);
}
template <typename T>
__device__ __forceinline__ typename Four<T>::Word raw_of(const pair32 *p) {
    const float2 a = parts(p[0]), b = parts(p[1]);
    const float f[8] = {a.x, a.y, b.x, b.y};
    Vec<T> v;
    v.set(f);
    if constexpr (sizeof(T) == 4) return v.raw;
    else return make_uint2(v.raw.x, v.raw.y);
}
template <int P>
__device__ __forceinline__ void floats_of(const float *f, pair32 *p) {
#pragma unroll
    for (int i = 0; i < P; i += 2) {
        const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(f + 2 * i);
        p[i] = u.x, p[i + 1] = u.y;
    }
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// gamma of queries and of keys
__device__ __forceinline__ void stage_gamma(const QkArgs &a, float (&to)[2][kMaxD]) {
    for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
        const float *from = i < a.d ? a.gamma_q : a.gamma_k;
        const int n = i < a.d ? i : i - a.d;
        to[i >= a.d][n] = from ? from[n] : 1.f;
    }
    __syncthreads();
}

constexpr int kHeads = 2;  // of a lane's, on their way at a time: the larger case above 40 us; one 56, three 40, four 43

template <typename T, bool INTERLEAVED, bool ALL, bool SMALL>
__global__ void __launch_bounds__(256, 4) qk_fwd_kernel(QkArgs a, Lanes k) {
    grid_wait();
    constexpr int V = 4, P = V / 2;
    using Word = typename Four<T>::Word;
    __shared__ alignas(16) float gamma[2][kMaxD];
    __shared__ float2 tables[8][kMaxD / 2];
    stage_gamma(a, gamma);
    Turns<T, INTERLEAVED, ALL> turns(a, k);
    const int group = threadIdx.x % 32 / k.lanes, groups = 32 / k.lanes, all = a.heads + a.kv;
    const long long items = (long long)a.rows * k.parts, step = (long long)gridDim.x * 8;
    for (long long item = (long long)blockIdx.x * 8 + threadIdx.x / 32; item < items; item += step) {
        const long long row = item / k.parts;
        const int h0 = (int)(item - row * k.parts) * k.heads, h1 = min(all, h0 + k.heads);
        const T *q = static_cast<const T *>(a.q) + row * a.ldq, *key = static_cast<const T *>(a.k) + row * a.ldk - (long long)a.heads * a.d;
        T *qo = static_cast<T *>(a.qo) + row * a.ldqo, *ko = static_cast<T *>(a.ko) + row * a.ldko - (long long)a.heads * a.d;
        bool made = false;
        for (int h = h0 + group; h - group < h1; h += kHeads * groups) {
            Word raw[kHeads][2];
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                const int n = h + i * groups;
                raw[i][0] = raw[i][1] = Word{};
                if (n < h1 && turns.on) {
                    const T *x = (n < a.heads ? q : key) + (long long)n * a.d;
                    raw[i][0] = *reinterpret_cast<const Word *>(x + turns.first);
                    raw[i][1] = *reinterpret_cast<const Word *>(x + turns.second);
                }
            }
            if (!made) turns.row(a, row, tables[threadIdx.x / 32]);
            made = true;
#pragma unroll
            for (int i = 0; i < kHeads; ++i) {
                const int n = h + i * groups;
                if (n - group >= h1) break;
                pair32 x[V], g[V], s = 0;
                pairs_of<T>(raw[i][0], x);
                pairs_of<T>(raw[i][1], x + P);
#pragma unroll
                for (int j = 0; j < V; ++j) s = fma2(x[j], x[j], s);
                const float2 f = parts(s);
                const float r = root<SMALL>(a, lanes_sum(f.x + f.y, k.lanes));
                if (n >= h1 || !turns.on) continue;
                floats_of<P>(&gamma[n >= a.heads][turns.first], g);
                floats_of<P>(&gamma[n >= a.heads][turns.second], g + P);
                const pair32 rr = pair_of(r, r);
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = mul2(mul2(x[j], rr), g[j]);
                turns.template apply<false>(a, x);
                T *y = (n < a.heads ? qo : ko) + (long long)n * a.d;
                *reinterpret_cast<Word *>(y + turns.first) = raw_of<T>(x);
                *reinterpret_cast<Word *>(y + turns.second) = raw_of<T>(x + P);
            }
        }
    }
}

// With n = R^T dy (turned back), g = gamma n and r = 1 / sqrt(mean x^2 + eps): dx = r g - x r^3 mean(g x), dgamma += n x r.  Both sums of a head are
// made at once.  A warp has either queries or keys, and keeps its share of the gradient of their gamma.
template <typename T, bool INTERLEAVED, bool ALL, bool SMALL>
__global__ void __launch_bounds__(256, 2) qk_bwd_kernel(QkArgs a, Lanes k) {
    grid_wait();
    constexpr int V = 4, P = V / 2, U = 4;
    using Word = typename Four<T>::Word;
    __shared__ alignas(16) float gamma[2][kMaxD];
    __shared__ float2 tables[8][kMaxD / 2];
    __shared__ float shares[8][kMaxD];
    stage_gamma(a, gamma);
    Turns<T, INTERLEAVED, ALL> turns(a, k);
    const int group = threadIdx.x % 32 / k.lanes, groups = 32 / k.lanes, w = threadIdx.x / 32;
    const bool keys = w >= k.warps;
    const int heads = keys ? a.kv : a.heads, mine = keys ? w - k.warps : w, warps = keys ? 8 - k.warps : k.warps;
    const long long ld = keys ? a.ldk : a.ldq, ldo = keys ? a.ldko : a.ldqo;
    const T *x0 = static_cast<const T *>(keys ? a.k : a.q), *dy0 = static_cast<const T *>(keys ? a.dko : a.dqo);
    T *dx0 = static_cast<T *>(keys ? a.dk : a.dq);
    pair32 sum[V] = {};
    const int parts_ = (heads + k.heads - 1) / k.heads;  // of a row
    const long long items = (long long)a.rows * parts_, step = (long long)gridDim.x * warps;
    for (long long item = (long long)blockIdx.x * warps + mine; item < items; item += step) {
        const long long row = item / parts_;
        const int h0 = (int)(item - row * parts_) * k.heads, h1 = min(heads, h0 + k.heads);
        bool made = false;
        for (int h = h0 + group; h - group < h1; h += U * groups) {
            Word xr[U][2], gr[U][2];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int n = h + i * groups;
                xr[i][0] = xr[i][1] = gr[i][0] = gr[i][1] = Word{};
                if (n < h1 && turns.on) {
                    const T *x = x0 + row * ld + (long long)n * a.d, *dy = dy0 + row * ldo + (long long)n * a.d;
                    xr[i][0] = *reinterpret_cast<const Word *>(x + turns.first);
                    xr[i][1] = *reinterpret_cast<const Word *>(x + turns.second);
                    gr[i][0] = *reinterpret_cast<const Word *>(dy + turns.first);
                    gr[i][1] = *reinterpret_cast<const Word *>(dy + turns.second);
                }
            }
            if (!made) turns.row(a, row, tables[w]);
            made = true;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int n = h + i * groups;
                if (n - group >= h1) break;
                pair32 x[V], g[V], s = 0, t = 0;
                pairs_of<T>(xr[i][0], x);
                pairs_of<T>(xr[i][1], x + P);
                pairs_of<T>(gr[i][0], g);
                pairs_of<T>(gr[i][1], g + P);
                turns.template apply<true>(a, g);
                pair32 gam[V];
                if (turns.on) {
                    floats_of<P>(&gamma[keys][turns.first], gam);
                    floats_of<P>(&gamma[keys][turns.second], gam + P);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) gam[j] = 0;
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    s = fma2(x[j], x[j], s);
                    t = fma2(mul2(g[j], x[j]), gam[j], t);
                }
                const float2 f = parts(s), u = parts(t);
                const float r = root<SMALL>(a, lanes_sum(f.x + f.y, k.lanes));
                const float m = -lanes_sum(u.x + u.y, k.lanes) * a.inv_d * r * r;
                if (n >= h1 || !turns.on) continue;
                const pair32 rr = pair_of(r, r), mm = pair_of(m, m);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    sum[j] = fma2(mul2(g[j], x[j]), rr, sum[j]);
                    g[j] = mul2(rr, fma2(x[j], mm, mul2(g[j], gam[j])));
                }
                T *dx = dx0 + row * ld + (long long)n * a.d;
                *reinterpret_cast<Word *>(dx + turns.first) = raw_of<T>(g);
                *reinterpret_cast<Word *>(dx + turns.second) = raw_of<T>(g + P);
            }
        }
    }
    if (!a.part) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float2 f = parts(sum[j]);
        for (int o = k.lanes; o < 32; o *= 2) {
            f.x += __shfl_xor_sync(0xffffffffu, f.x, o);
            f.y += __shfl_xor_sync(0xffffffffu, f.y, o);
        }
        if (group == 0 && turns.on) {
            float *to = &shares[w][j < P ? turns.first + 2 * j : turns.second + 2 * (j - P)];
            to[0] = f.x, to[1] = f.y;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
        const int which = i >= a.d, n = which ? i - a.d : i;
        float s = 0.f;
        for (int v = which ? k.warps : 0; v < (which ? 8 : k.warps); ++v) s += shares[v][n];
        a.part[((size_t)blockIdx.x * 2 + which) * a.d + n] = s;
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
    a.inv_d = 1.f / (float)d->d;
    return a;
}

// Blocks of eight warps, each with a head, or with the lanes' heads of a row: by sizes alone, so that the order of the sums goes by them.
int blocks_of(long long items, int per_sm) {
    const long long all = (items + 7) / 8;
    return (int)(all < per_sm * 148 ? all : per_sm * 148);
}
int any_blocks(const ppo_qk_norm_desc *d) { return blocks_of((long long)d->rows * (d->heads + d->kv_heads), 4); }

// Whether every row is made of whole, aligned vectors, and pairs lie in two of a lane's.
bool vectors(const ppo_qk_norm_desc *d, std::initializer_list<const void *> ps) {
    constexpr int V = 4;
    return d->d % (2 * V) == 0 && (d->interleaved || d->pairs % V == 0) && d->ldq % V == 0 && d->ldk % V == 0 && d->ldqo % V == 0 && d->ldko % V == 0 &&
           !misaligned(ps, V * elem_bytes(d->dtype));
}
// Rows are taken whole, as long as they give every SM `warps` warps; fewer rows are dealt out by as many heads as the lanes of a warp take at once.
Lanes lanes_of(const ppo_qk_norm_desc *d, int warps) {
    const int all = d->heads + d->kv_heads;
    Lanes k = {1, d->d / 8, 1, all};
    while (k.lanes < k.slots) k.lanes *= 2;
    const int side = 32 / k.lanes, most = ppo_cdiv(all, side);
    long long want = ((long long)warps * 148 + d->rows - 1) / d->rows;
    k.parts = (int)(want < most ? want : most);
    k.heads = ppo_cdiv(ppo_cdiv(all, k.parts), side) * side;
    k.parts = ppo_cdiv(all, k.heads);
    k.warps = (8 * d->heads + all / 2) / all;
    k.warps = k.warps < 1 ? 1 : k.warps > 7 ? 7 : k.warps;
    return k;
}
// fn(T{}, interleaved, whole heads turned, eps below the normal numbers)
template <typename F>
int with_order(const ppo_qk_norm_desc *d, float eps, F &&fn) {
    const std::true_type yes;
    const std::false_type no;
    return with_elem(d->dtype, [&](auto t) -> int {
        const auto ordered = [&](auto all, auto small) -> int { return d->interleaved ? fn(t, yes, all, small) : fn(t, no, all, small); };
        if (eps < FLT_MIN) return ordered(no, yes);
        return 2 * d->pairs == d->d ? ordered(yes, no) : ordered(no, no);
    });
}

}  // namespace

extern "C" size_t ppo_qk_norm_rotate_workspace_bytes(const ppo_qk_norm_desc *d) {
    return check(d) == PPO_OK ? (size_t)4 * 148 * 2 * d->d * sizeof(float) : 0;
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
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!vectors(d, {q, k, q_out, k_out}))
        return with_elem(d->dtype, [&](auto t) { return ppo_launch(qk_fwd_any_kernel<decltype(t)>, dim3(any_blocks(d)), dim3(256), 0, st, a); });
    const Lanes l = lanes_of(d, 32);
    return with_order(d, eps, [&](auto t, auto order, auto all, auto small) {
        return ppo_launch(qk_fwd_kernel<decltype(t), decltype(order)::value, decltype(all)::value, decltype(small)::value>,
                          dim3(blocks_of((long long)d->rows * l.parts, 4)), dim3(256), 0, st, a, l);
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
    int blocks = any_blocks(d);
    if (vectors(d, {q, k, dq_out, dk_out, dq, dk})) {
        const Lanes l = lanes_of(d, 32);
        blocks = blocks_of((long long)d->rows * l.parts, 2);
        PPO_TRY(with_order(d, eps, [&](auto t, auto order, auto all, auto small) {
            return ppo_launch(qk_bwd_kernel<decltype(t), decltype(order)::value, decltype(all)::value, decltype(small)::value>, dim3(blocks), dim3(256), 0, st, a,
                              l);
        }));
    } else {
        PPO_TRY(with_elem(d->dtype, [&](auto t) { return ppo_launch(qk_bwd_any_kernel<decltype(t)>, dim3(blocks), dim3(256), 0, st, a); }));
    }
    return params ? ppo_param_sum(a.part, blocks, {{dgamma_q, dgamma_k, nullptr}, {d->d, d->d, 0}}, accumulate, st) : PPO_OK;
}
