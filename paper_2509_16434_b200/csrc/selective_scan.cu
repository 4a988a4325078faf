// Selective scan: states whose decay and input the data choose, and its gradients.
//
// h_t = exp(d_t A) h_{t-1} + d_t x_t B_t: one exponential and four multiply-adds for each element of a state and step, against 8 bytes
// for each channel and step in 16 bits: with 16 elements a channel the exponentials (16 a clock and SM) bound it, not memory.
//
// A block of four warps takes a tile of channels of one env through the steps, 16 at a time: step sizes and inputs are made once for each
// channel and step and left in shared memory, with the rows of B and C; then every thread goes through the steps with NPT elements of the states
// of four neighbouring channels in registers, packed arithmetic on two channels at a time; sums over the elements of a state go over the NL
// lanes that share its channel, halving what each holds (three shuffles a step for four channels).  States, sums and arithmetic in 32 bits.
#include "approx.cuh"
#include "elem.cuh"
#include "pair32.cuh"
#include "param_sum.cuh"

namespace {

constexpr int kMaxN = 64, kThreads = 128, kSteps = 16;

struct ScanArgs {
    const void *x, *dt, *B, *C, *z, *dy;
    const float *A, *D, *bias, *state_in, *dstate_out;
    const uint8_t *done;
    void *y, *dx, *ddt, *dB, *dC, *dz;
    float *state_out, *dstate_in;
    long long ldx, lddt, ldb, ldc, ldz, ldy;
    int T, Be, channels, N, groups, per, softplus;  // per: channels of a group
    int tiles, group_tiles;                         // tiles of channels, in all and of a group
    int len, nseg;                                  // steps of a segment
    // Of every segment, env and tile, as the threads of a tile hold them: the states it ends with (starting from zeros, but for the first one;
    // in the last one's place the state that comes in) and the gradients it hands to the steps in front (getting zeros; in the first
    // one's place the gradient of the state that is left); what its step sizes add up to for each channel, and whether a flag is set in it.
    float *seg, *back, *sum;
    int *cut;
    float *mark;  // the states in front of every fourth step, [ceil(T / 4)][Be][tiles] as the threads hold them
    float *few;   // shares of the gradients of B and C, [group_tiles][T * Be][groups][2][NP]
    float *part;  // shares of the gradients of A, D and dt_bias, [parts][channels * (N + 2)]
    int parts;
};

__device__ __forceinline__ pair32 twice(float a) { return pair_of(a, a); }
__device__ __forceinline__ pair32 exp2_pair(pair32 p) {
    const float2 f = parts(p);
    return pair_of(exp2_fast(f.x), exp2_fast(f.y));
}

// Sums of V values over LANES lanes, STRIDE apart: halves go to the lanes' halves as long as there are values, lane bit by lane bit from the
// highest; a lane is left with max(1, V / LANES) of them in v[0 ..].  index() says which.
template <int V, int LANES, int STRIDE>
__device__ __forceinline__ void spread_sum(float (&v)[V], int lane) {
    if constexpr (LANES > 1) {
        constexpr int O = LANES / 2 * STRIDE;
        if constexpr (V > 1) {
            const bool up = lane & O;
            float half[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float give = up ? v[i] : v[i + V / 2];
                half[i] = (up ? v[i + V / 2] : v[i]) + __shfl_xor_sync(0xffffffffu, give, O);
            }
            spread_sum<V / 2, LANES / 2, STRIDE>(half, lane);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) v[i] = half[i];
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], O);
            spread_sum<V, LANES / 2, STRIDE>(v, lane);
        }
    }
}
// The first of a lane's values after spread_sum: V values halved over lanes numbered l of LANES.
template <int V, int LANES>
__device__ __forceinline__ int spread_first(int l) {
    if constexpr (V > 1 && LANES > 1) return (l & (LANES / 2) ? V / 2 : 0) + spread_first<V / 2, LANES / 2>(l);
    else return 0;
}

// NL lanes share four channels and hold NPT elements each of their states.
template <int NPT, int NL>
struct Shape {
    static constexpr int NP = NPT * NL, GROUPS = 32 / NL, CT = 4 * GROUPS * (kThreads / 32);
};

// What a block works on: a tile of channels of one env over steps t0 .. t1 - 1.
struct Work {
    int tile, e, seg, t0, t1, group, c0, c1;  // channels c0 .. c1 - 1 of the group
};
template <int CT>
__device__ __forceinline__ Work work_of(const ScanArgs &a, int tile, long long item) {
    Work w;
    w.tile = tile;
    w.seg = (int)(item / a.Be);
    w.e = (int)(item - (long long)w.seg * a.Be);
    w.t0 = w.seg * a.len;
    w.t1 = min(a.T, w.t0 + a.len);
    w.group = tile / a.group_tiles;
    w.c0 = w.group * a.per + (tile - w.group * a.group_tiles) * CT;
    w.c1 = min((w.group + 1) * a.per, w.c0 + CT);
    return w;
}

// kSteps rows of a tile's channels on their way from memory: vectors of V elements, dealt out to the threads.
template <typename T, int CT, bool VEC>
struct Rows {
    static constexpr int V = VEC ? 16 / (int)sizeof(T) : 1, COLS = CT / V, PASSES = (kSteps * COLS + kThreads - 1) / kThreads;
    using Raw = std::conditional_t<VEC, uint4, T>;
    Raw raw[PASSES];
    static __device__ __forceinline__ int row(int i) { return (threadIdx.x + i * kThreads) / COLS; }
    static __device__ __forceinline__ int col(int i) { return (threadIdx.x + i * kThreads) % COLS * V; }
    // p: the tile's first channel in the env's row of step t
    __device__ __forceinline__ void fetch(const T *p, long long step, int rows, int cols) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (row(i) < min(rows, kSteps) && col(i) < cols) raw[i] = *reinterpret_cast<const Raw *>(p + row(i) * step + col(i));
    }
    __device__ __forceinline__ void get(int i, float (&v)[V]) const {
        if constexpr (VEC) {
            Vec<T> x;
            x.raw = raw[i];
            x.get(v);
        } else {
            v[0] = to_f32(raw[i]);
        }
    }
    static __device__ __forceinline__ void put(T *p, const float (&v)[V]) {
        if constexpr (VEC) {
            Vec<T> x;
            x.set(v);
            *reinterpret_cast<uint4 *>(p) = x.raw;
        } else {
            *p = from_f32<T>(v[0]);
        }
    }
};
template <int V>
__device__ __forceinline__ void put_floats(float *p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}
template <int V>
__device__ __forceinline__ void get_floats(const float *p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = *p;
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(p + i);
            v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
        }
    }
}

// The rows of B or C, padded with zeros to NP elements, each of them twice, as packed arithmetic on two channels takes it; zeros behind the
// last step.
template <typename T, int NP>
__device__ __forceinline__ void stage_few(float2 (&to)[kSteps][NP], const T *from, long long step, int rows, int N) {
    for (int i = threadIdx.x; i < kSteps * NP; i += kThreads) {
        const int t = i / NP, n = i % NP;
        const float v = t < rows && n < N ? to_f32(from[t * step + n]) : 0.f;
        to[t][n] = make_float2(v, v);
    }
}
// Of the tile's channels; zeros where there are none.
template <int CT>
__device__ __forceinline__ void stage_channels(float (&to)[CT], const float *from, const Work &w) {
    for (int i = threadIdx.x; i < CT; i += kThreads) to[i] = from && w.c0 + i < w.c1 ? from[w.c0 + i] : 0.f;
}
// Bit r: the flag of step t + r, 0 behind the last one.
__device__ __forceinline__ uint32_t flags_of(const ScanArgs &a, int e, int t, int rows) {
    const int r = threadIdx.x % 32;
    return a.done ? __ballot_sync(0xffffffffu, r < min(rows, kSteps) && t + r >= 0 && a.done[(long long)(t + r) * a.Be + e]) : 0u;
}

// NPT elements of four channels' states, [e][channel][N] in memory; zeros where there are none.
template <int NPT>
__device__ __forceinline__ void load_state(const float *from, const ScanArgs &a, int e, int c, int c1, int n0, float (&h)[4][NPT]) {
    const bool whole = NPT == 4 && a.N % 4 == 0 && (reinterpret_cast<uintptr_t>(from) & 15) == 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int n = 0; n < NPT; ++n) h[j][n] = 0.f;
        if (!from || c + j >= c1) continue;
        const float *p = from + ((long long)e * a.channels + c + j) * a.N + n0;
        if (whole) {
            if constexpr (NPT == 4) {
                if (n0 < a.N) {
                    const float4 f = *reinterpret_cast<const float4 *>(p);
                    h[j][0] = f.x, h[j][1] = f.y, h[j][2] = f.z, h[j][3] = f.w;
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < NPT; ++n)
                if (n0 + n < a.N) h[j][n] = p[n];
        }
    }
}
template <int NPT>
__device__ __forceinline__ void store_state(float *to, const ScanArgs &a, int e, int c, int c1, int n0, const float (&h)[4][NPT]) {
    const bool whole = NPT == 4 && a.N % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & 15) == 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (c + j >= c1) break;
        float *p = to + ((long long)e * a.channels + c + j) * a.N + n0;
        if (whole) {
            if (n0 < a.N) *reinterpret_cast<float4 *>(p) = make_float4(h[j][0], h[j][1], h[j][2], h[j][3]);
        } else {
#pragma unroll
            for (int n = 0; n < NPT; ++n)
                if (n0 + n < a.N) p[n] = h[j][n];
        }
    }
}
// The same as the threads hold them.
template <int NPT>
__device__ __forceinline__ void load_held(const float *from, long long tile, float (&h)[4][NPT]) {
    const float *p = from + tile * (kThreads * 4 * NPT) + threadIdx.x * 4;
#pragma unroll
    for (int n = 0; n < NPT; ++n) {
        const float4 f = *reinterpret_cast<const float4 *>(p + n * kThreads * 4);
        h[0][n] = f.x, h[1][n] = f.y, h[2][n] = f.z, h[3][n] = f.w;
    }
}
template <int NPT>
__device__ __forceinline__ void store_held(float *to, long long tile, const float (&h)[4][NPT]) {
    float *p = to + tile * (kThreads * 4 * NPT) + threadIdx.x * 4;
#pragma unroll
    for (int n = 0; n < NPT; ++n) *reinterpret_cast<float4 *>(p + n * kThreads * 4) = make_float4(h[0][n], h[1][n], h[2][n], h[3][n]);
}
template <int NPT>
__device__ __forceinline__ void pack(const float (&h)[4][NPT], pair32 (&p)[NPT][2]) {
#pragma unroll
    for (int n = 0; n < NPT; ++n) p[n][0] = pair_of(h[0][n], h[1][n]), p[n][1] = pair_of(h[2][n], h[3][n]);
}
template <int NPT>
__device__ __forceinline__ void unpack(const pair32 (&p)[NPT][2], float (&h)[4][NPT]) {
#pragma unroll
    for (int n = 0; n < NPT; ++n) {
        const float2 u = parts(p[n][0]), v = parts(p[n][1]);
        h[0][n] = u.x, h[1][n] = u.y, h[2][n] = v.x, h[3][n] = v.y;
    }
}
__device__ __forceinline__ void load_pairs(const float *p, pair32 (&v)[2]) {
    const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p);
    v[0] = u.x, v[1] = u.y;
}
template <int NPT>
__device__ __forceinline__ void load_few(const float2 *p, pair32 (&v)[NPT]) {
    if constexpr (NPT % 2 == 0) {
#pragma unroll
        for (int n = 0; n < NPT; n += 2) {
            const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p + n);
            v[n] = u.x, v[n + 1] = u.y;
        }
    } else {
#pragma unroll
        for (int n = 0; n < NPT; ++n) v[n] = *reinterpret_cast<const pair32 *>(p + n);
    }
}

// exp2(A sum of a segment's step sizes) h + add, or add alone behind a flag.
template <int NPT>
__device__ __forceinline__ void through(const ScanArgs &a, const Work &w, int s, int c, const float (&A)[4][NPT], const float *from, float (&h)[4][NPT]) {
    const long long at = (long long)s * a.Be + w.e;
    float add[4][NPT];
    load_held<NPT>(from, at * a.tiles + w.tile, add);
    const bool cut = a.cut[at];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float d = c + j < w.c1 ? a.sum[at * a.channels + c + j] : 0.f;
#pragma unroll
        for (int n = 0; n < NPT; ++n) h[j][n] = cut ? add[j][n] : fmaf(exp2_fast(d * A[j][n]), h[j][n], add[j][n]);
    }
}
// What a segment starts from: the state that comes in, or what the first segment ends with, taken through the segments in between.
template <int NPT>
__device__ __forceinline__ void start_of(const ScanArgs &a, const Work &w, int c, const float (&A)[4][NPT], float (&h)[4][NPT]) {
    const long long at = (long long)(w.seg == 0 ? a.nseg - 1 : 0) * a.Be + w.e;
    load_held<NPT>(a.seg, at * a.tiles + w.tile, h);
    for (int s = 1; s < w.seg; ++s) through<NPT>(a, w, s, c, A, a.seg, h);
}
// The gradient that a segment gets of the state it leaves.
template <int NPT>
__device__ __forceinline__ void end_of(const ScanArgs &a, const Work &w, int c, const float (&A)[4][NPT], float (&g)[4][NPT]) {
    load_held<NPT>(a.back, (long long)w.e * a.tiles + w.tile, g);
    for (int s = a.nseg - 1; s > w.seg; --s) through<NPT>(a, w, s, c, A, a.back, g);
}

enum Mode {
    OUTPUT,  // y and the state that is left
    ENDS,    // what each segment ends with
    BOTH,    // that, and the gradients it hands to the steps in front
    MARKS    // the states in front of every fourth step
};

template <typename T, int NPT, int NL, int MODE, bool VEC>
__global__ void __launch_bounds__(kThreads, MODE == BOTH ? 3 : 5) scan_kernel(ScanArgs a) {
    grid_wait();
    using S = Shape<NPT, NL>;
    constexpr int CT = S::CT, NP = S::NP;
    constexpr bool WITH_C = MODE == OUTPUT || MODE == BOTH, WITH_DY = MODE == BOTH;
    using R = Rows<T, CT, VEC>;
    __shared__ alignas(16) float sd[kSteps][CT], su[kSteps][CT], sg[WITH_DY ? kSteps : 1][CT], sD[CT], sbias[CT];
    __shared__ alignas(16) float2 sB[kSteps][NP], sC[kSteps][WITH_C ? NP : 1];
    const Work w = work_of<CT>(a, blockIdx.x % a.tiles, blockIdx.x / a.tiles);
    const int lane = threadIdx.x % 32, ln = lane % NL, c = w.c0 + (threadIdx.x / 32 * S::GROUPS + lane / NL) * 4, n0 = ln * NPT, local = c - w.c0;
    const int cols = w.c1 - w.c0;
    const long long sx = a.Be * a.ldx, st = a.Be * a.lddt, sb = a.Be * a.ldb, sc = a.Be * a.ldc, sz = a.Be * a.ldz, sy = a.Be * a.ldy;
    const T *x = static_cast<const T *>(a.x) + w.e * a.ldx + w.c0, *dt = static_cast<const T *>(a.dt) + w.e * a.lddt + w.c0;
    const T *B = static_cast<const T *>(a.B) + w.e * a.ldb + (long long)w.group * a.N, *C = static_cast<const T *>(a.C) + w.e * a.ldc + (long long)w.group * a.N;
    const T *z = a.z ? static_cast<const T *>(a.z) + w.e * a.ldz + w.c0 : nullptr;
    const T *dy = WITH_DY ? static_cast<const T *>(a.dy) + w.e * a.ldy + w.c0 : nullptr;

    pair32 A[NPT][2], h[NPT][2], P[WITH_DY ? NPT : 1][2], G[WITH_DY ? NPT : 1][2];
    const long long held = ((long long)w.seg * a.Be + w.e) * a.tiles + w.tile;
    {
        float Af[4][NPT], f[4][NPT] = {};
        load_state<NPT>(a.A, a, 0, c, w.c1, n0, Af);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NPT; ++n) Af[j][n] *= kLog2e;
        pack<NPT>(Af, A);
        if (MODE == ENDS || MODE == BOTH || a.nseg == 1) {
            if (w.seg == 0) {
                load_state<NPT>(a.state_in, a, w.e, c, w.c1, n0, f);
                if (a.nseg > 1) store_held<NPT>(a.seg, held + (long long)(a.nseg - 1) * a.Be * a.tiles, f);
            }
        } else {
            start_of<NPT>(a, w, c, Af, f);
        }
        pack<NPT>(f, h);
        if constexpr (WITH_DY) {
#pragma unroll
            for (int n = 0; n < NPT; ++n) P[n][0] = P[n][1] = twice(1.f), G[n][0] = G[n][1] = 0;
        }
    }
    R rx, rt;
    rx.fetch(x + w.t0 * sx, sx, w.t1 - w.t0, cols);
    rt.fetch(dt + w.t0 * st, st, w.t1 - w.t0, cols);
    stage_channels(sbias, a.bias, w);
    if constexpr (MODE == OUTPUT) stage_channels(sD, a.D, w);
    __syncthreads();
    float total[4] = {};
    bool cut = false;
    for (int t = w.t0; t < w.t1; t += kSteps) {
        const int rows = w.t1 - t;
        R rg, rz;
        if constexpr (WITH_DY) {
            rg.fetch(dy + t * sy, sy, rows, cols);
            if (z) rz.fetch(z + t * sz, sz, rows, cols);
        }
#pragma unroll
        for (int i = 0; i < R::PASSES; ++i) {
            const int r = R::row(i), l = R::col(i);
            if (r >= kSteps) break;
            float d[R::V] = {}, u[R::V] = {}, g[R::V] = {};
            if (r < rows && l < cols) {
                float b[R::V];
                rt.get(i, d);
                rx.get(i, u);
                get_floats(&sbias[l], b);
#pragma unroll
                for (int v = 0; v < R::V; ++v) {
                    d[v] += b[v];
                    if (a.softplus) d[v] = softplus_fast(d[v]);
                    u[v] *= d[v];
                }
                if constexpr (WITH_DY) {
                    rg.get(i, g);
                    if (z) {
                        float f[R::V];
                        rz.get(i, f);
#pragma unroll
                        for (int v = 0; v < R::V; ++v) g[v] *= f[v] * sigmoid_fast(f[v]);
                    }
                }
            }
            put_floats(&sd[r][l], d);
            put_floats(&su[r][l], u);
            if constexpr (WITH_DY) put_floats(&sg[r][l], g);
        }
        stage_few<T, NP>(sB, B + t * sb, sb, rows, a.N);
        if constexpr (WITH_C) stage_few<T, NP>(sC, C + t * sc, sc, rows, a.N);
        const uint32_t flag = flags_of(a, w.e, t, rows);
        __syncthreads();
        if (t + kSteps < w.t1) {
            rx.fetch(x + (t + kSteps) * sx, sx, rows - kSteps, cols);
            rt.fetch(dt + (t + kSteps) * st, st, rows - kSteps, cols);
        }
        for (int s = 0; s < kSteps && s < rows; s += 4) {
            if constexpr (MODE == MARKS) {
                float f[4][NPT];
                unpack<NPT>(h, f);
                store_held<NPT>(a.mark, ((long long)((t + s) / 4) * a.Be + w.e) * a.tiles + w.tile, f);
            }
            float out[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                pair32 d[2], u[2], g[2], acc[2] = {0, 0};
                pair32 b[NPT], cc[NPT];
                load_pairs(&sd[s + k][local], d);
                load_pairs(&su[s + k][local], u);
                load_few<NPT>(&sB[s + k][n0], b);
                if constexpr (WITH_C) load_few<NPT>(&sC[s + k][n0], cc);
                if constexpr (WITH_DY) load_pairs(&sg[s + k][local], g);
#pragma unroll
                for (int n = 0; n < NPT; ++n)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const pair32 f = exp2_pair(mul2(d[p], A[n][p]));
                        h[n][p] = fma2(f, h[n][p], mul2(u[p], b[n]));
                        if constexpr (MODE == OUTPUT) acc[p] = fma2(cc[n], h[n][p], acc[p]);
                        if constexpr (WITH_DY) {
                            P[n][p] = mul2(P[n][p], f);
                            if (!cut) G[n][p] = fma2(mul2(P[n][p], g[p]), cc[n], G[n][p]);
                        }
                    }
                if constexpr (MODE == OUTPUT) {
                    const float2 p = parts(acc[0]), q = parts(acc[1]);
                    out[4 * k] = p.x, out[4 * k + 1] = p.y, out[4 * k + 2] = q.x, out[4 * k + 3] = q.y;
                }
                if constexpr (MODE == ENDS || MODE == BOTH) {
                    const float2 p = parts(d[0]), q = parts(d[1]);
                    total[0] += p.x, total[1] += p.y, total[2] += q.x, total[3] += q.y;
                }
                if (flag >> (s + k) & 1) {
                    cut = true;
#pragma unroll
                    for (int n = 0; n < NPT; ++n) h[n][0] = h[n][1] = 0;
                }
            }
            if constexpr (MODE == OUTPUT) {
                // every lane of the channels has read the step sizes of these steps: the sums take their place
                spread_sum<16, NL, 1>(out, lane);
                constexpr int LEFT = 16 / NL;
                const int first = spread_first<16, NL>(ln);
                float *to = &sd[s + first / 4][local + first % 4];
                if constexpr (LEFT == 4) *reinterpret_cast<float4 *>(to) = make_float4(out[0], out[1], out[2], out[3]);
                else if constexpr (LEFT == 2) *reinterpret_cast<float2 *>(to) = make_float2(out[0], out[1]);
                else *to = out[0];
            }
        }
        __syncthreads();
        if constexpr (MODE == OUTPUT) {
            T *y = static_cast<T *>(a.y) + w.e * a.ldy + w.c0;
            R again, gate;
            again.fetch(x + t * sx, sx, rows, cols);
            if (z) gate.fetch(z + t * sz, sz, rows, cols);
#pragma unroll
            for (int i = 0; i < R::PASSES; ++i) {
                const int r = R::row(i), l = R::col(i);
                if (r >= kSteps || r >= rows || l >= cols) continue;
                float o[R::V], v[R::V];
                get_floats(&sd[r][l], o);
                if (a.D) {
                    float D[R::V];
                    again.get(i, v);
                    get_floats(&sD[l], D);
#pragma unroll
                    for (int k = 0; k < R::V; ++k) o[k] = fmaf(D[k], v[k], o[k]);
                }
                if (z) {
                    gate.get(i, v);
#pragma unroll
                    for (int k = 0; k < R::V; ++k) o[k] *= v[k] * sigmoid_fast(v[k]);
                }
                R::put(y + (t + r) * sy + l, o);
            }
            __syncthreads();
        }
    }
    float f[4][NPT];
    unpack<NPT>(h, f);
    if constexpr (MODE == OUTPUT) {
        if (a.state_out && w.t1 == a.T) store_state<NPT>(a.state_out, a, w.e, c, w.c1, n0, f);
    }
    if constexpr (MODE == ENDS || MODE == BOTH) {
        const long long at = (long long)w.seg * a.Be + w.e;
        if (w.seg < a.nseg - 1) store_held<NPT>(a.seg, held, f);
        if (ln == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < w.c1) a.sum[at * a.channels + c + j] = total[j];
        }
        if (threadIdx.x == 0 && w.tile == 0) a.cut[at] = cut;
    }
    if constexpr (MODE == BOTH) {
        if (w.seg > 0) unpack<NPT>(G, f);
        else load_state<NPT>(a.dstate_out, a, w.e, c, w.c1, n0, f);
        store_held<NPT>(a.back, held, f);
    }
}

// Gradients.  Per step, with g = dL/dh_t and dv = dL/dy silu(z):
//   g_t = C_t dv_t + (nothing where done[t] is set, else) exp(d_{t+1} A) g_{t+1},   q = g_t exp(d_t A) h'_{t-1}
//   dC = sum_c dv h,  dB = sum_c g d x,  dx = D dv + d sum_n g B,  dd = x sum_n g B + sum_n q A,  dA += q d
// Four steps at a time, backwards: from the states in front of them forwards once more, which leaves the factors and exp(d A) h' of the
// four steps in registers (and y and the sums of dC on the way), then backwards over these.  A block goes through as many envs, or
// segments, as fall to it and keeps its shares of the parameters' gradients.
// A long sum as two numbers: what hi rounds away stays in lo (Knuth's error of a sum).
__device__ __forceinline__ void add_to(float &hi, float &lo, float v) {
    const float sum = __fadd_rn(hi, v), w = __fsub_rn(sum, hi);
    lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(sum, w)), __fsub_rn(v, w));
    hi = sum;
}

template <typename T, int NL, bool VEC>
struct GradShared {
    static constexpr int CT = Shape<4, NL>::CT, NP = Shape<4, NL>::NP;
    float sd[kSteps][CT], su[kSteps][CT], sg[kSteps][CT], sy[kSteps][CT], sD[CT], sbias[CT];
    float2 sB[kSteps][NP], sC[kSteps][NP];
    float few[kThreads / 32][kSteps][2 * NP];
    float mark[4][4][kThreads * 4];
    float dA[2][16][kThreads], kept[2][2][Rows<T, CT, VEC>::V][kThreads];  // [..][2]: hi and lo of the sums
};

__device__ __forceinline__ void copy_async(float *to, const float *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

template <typename T, int NL, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) scan_bwd_kernel(ScanArgs a) {
    grid_wait();
    constexpr int NPT = 4;
    using S = Shape<NPT, NL>;
    constexpr int CT = S::CT, NP = S::NP, GROUPS = S::GROUPS;
    using R = Rows<T, CT, VEC>;
    extern __shared__ __align__(16) char smem[];
    GradShared<T, NL, VEC> &s = *reinterpret_cast<GradShared<T, NL, VEC> *>(smem);
    const int tile = blockIdx.x % a.tiles, slice = blockIdx.x / a.tiles;
    const int lane = threadIdx.x % 32, ln = lane % NL, warp = threadIdx.x / 32, n0 = ln * NPT, local = (warp * GROUPS + lane / NL) * 4;
    Work w = work_of<CT>(a, tile, 0);
    const int c = w.c0 + local, cols = w.c1 - w.c0;
    const long long sx = a.Be * a.ldx, st = a.Be * a.lddt, sb = a.Be * a.ldb, sc = a.Be * a.ldc, sz = a.Be * a.ldz, sy = a.Be * a.ldy;
    pair32 A[NPT][2], g[NPT][2], dA[NPT][2];
    {
        float f[4][NPT];
        load_state<NPT>(a.A, a, 0, c, w.c1, n0, f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NPT; ++n) f[j][n] *= kLog2e;
        pack<NPT>(f, A);
#pragma unroll
        for (int n = 0; n < NPT; ++n) dA[n][0] = dA[n][1] = 0;
    }
    stage_channels(s.sD, a.D, w);
    stage_channels(s.sbias, a.bias, w);
#pragma unroll
    for (int v = 0; v < R::V; ++v)
#pragma unroll
        for (int k = 0; k < 4; ++k) s.kept[k / 2][k % 2][v][threadIdx.x] = 0.f;
#pragma unroll
    for (int n = 0; n < 16; ++n) s.dA[0][n][threadIdx.x] = s.dA[1][n][threadIdx.x] = 0.f;

    const long long items = (long long)a.Be * a.nseg;
    for (long long item = slice; item < items; item += a.parts) {
        w = work_of<CT>(a, tile, item);
        const T *x = static_cast<const T *>(a.x) + w.e * a.ldx + w.c0, *dt = static_cast<const T *>(a.dt) + w.e * a.lddt + w.c0;
        const T *B = static_cast<const T *>(a.B) + w.e * a.ldb + (long long)w.group * a.N, *C = static_cast<const T *>(a.C) + w.e * a.ldc + (long long)w.group * a.N;
        const T *z = a.z ? static_cast<const T *>(a.z) + w.e * a.ldz + w.c0 : nullptr, *dy = static_cast<const T *>(a.dy) + w.e * a.ldy + w.c0;
        {
            float f[4][NPT], Af[4][NPT];
            if (a.nseg == 1) {
                load_state<NPT>(a.dstate_out, a, w.e, c, w.c1, n0, f);
            } else {
                unpack<NPT>(A, Af);
                end_of<NPT>(a, w, c, Af, f);
            }
            pack<NPT>(f, g);
        }
        for (int t = w.t0 + (w.t1 - 1 - w.t0) / kSteps * kSteps; t >= w.t0; t -= kSteps) {
            const int rows = w.t1 - t;
            const uint32_t flag = flags_of(a, w.e, t, rows);
            __syncthreads();  // the tile behind is done with
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                if (4 * m >= rows) break;
                const float *from = a.mark + (((long long)(t / 4 + m) * a.Be + w.e) * a.tiles + tile) * (kThreads * 16) + threadIdx.x * 4;
#pragma unroll
                for (int n = 0; n < NPT; ++n) copy_async(&s.mark[m][n][threadIdx.x * 4], from + n * kThreads * 4);
            }
            {
                R rx, rt, rg, rz;
                rx.fetch(x + t * sx, sx, rows, cols);
                rt.fetch(dt + t * st, st, rows, cols);
                rg.fetch(dy + t * sy, sy, rows, cols);
                if (z) rz.fetch(z + t * sz, sz, rows, cols);
                stage_few<T, NP>(s.sB, B + t * sb, sb, rows, a.N);
                stage_few<T, NP>(s.sC, C + t * sc, sc, rows, a.N);
#pragma unroll
                for (int i = 0; i < R::PASSES; ++i) {
                    const int r = R::row(i), l = R::col(i);
                    if (r >= kSteps) break;
                    float d[R::V] = {}, u[R::V] = {}, v[R::V] = {};
                    if (r < rows && l < cols) {
                        rt.get(i, d);
                        rx.get(i, u);
                        rg.get(i, v);
                        float b[R::V];
                        get_floats(&s.sbias[l], b);
#pragma unroll
                        for (int k = 0; k < R::V; ++k) {
                            d[k] += b[k];
                            if (a.softplus) d[k] = softplus_fast(d[k]);
                            u[k] *= d[k];
                        }
                        if (z) {
                            float f[R::V];
                            rz.get(i, f);
#pragma unroll
                            for (int k = 0; k < R::V; ++k) v[k] *= f[k] * sigmoid_fast(f[k]);
                        }
                    }
                    put_floats(&s.sd[r][l], d);
                    put_floats(&s.su[r][l], u);
                    put_floats(&s.sg[r][l], v);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");  // a thread reads what it copied itself
            __syncthreads();
#pragma unroll 1
            for (int m = (min(rows, kSteps) - 1) / 4; m >= 0; --m) {
                const int r0 = 4 * m;
                pair32 f[4][NPT][2], q[4][NPT][2];  // of each step the factors, and these times the state in front
                {
                    pair32 h[NPT][2];
#pragma unroll
                    for (int n = 0; n < NPT; ++n) load_pairs(&s.mark[m][n][threadIdx.x * 4], h[n]);
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        float ys[8], cs[8];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int r = r0 + k + i;
                            pair32 d[2], u[2], v[2], acc[2] = {0, 0};
                            pair32 b[NPT], cc[NPT];
                            load_pairs(&s.sd[r][local], d);
                            load_pairs(&s.su[r][local], u);
                            load_pairs(&s.sg[r][local], v);
                            load_few<NPT>(&s.sB[r][n0], b);
                            load_few<NPT>(&s.sC[r][n0], cc);
                            if (k + i > 0 && flag >> (r - 1) & 1) {
#pragma unroll
                                for (int n = 0; n < NPT; ++n) h[n][0] = h[n][1] = 0;
                            }
#pragma unroll
                            for (int n = 0; n < NPT; ++n) {
                                pair32 sum = 0;
#pragma unroll
                                for (int p = 0; p < 2; ++p) {
                                    const pair32 e = exp2_pair(mul2(d[p], A[n][p])), qq = mul2(e, h[n][p]);
                                    f[k + i][n][p] = e;
                                    q[k + i][n][p] = qq;
                                    h[n][p] = fma2(u[p], b[n], qq);
                                    acc[p] = fma2(cc[n], h[n][p], acc[p]);
                                    sum = fma2(v[p], h[n][p], sum);
                                }
                                const float2 e = parts(sum);
                                cs[4 * i + n] = e.x + e.y;
                            }
                            const float2 e = parts(acc[0]), o = parts(acc[1]);
                            ys[4 * i] = e.x, ys[4 * i + 1] = e.y, ys[4 * i + 2] = o.x, ys[4 * i + 3] = o.y;
                        }
                        spread_sum<8, NL, 1>(ys, lane);
                        spread_sum<8, GROUPS, NL>(cs, lane);
                        int at = spread_first<8, NL>(ln);
#pragma unroll
                        for (int i = 0; i < (NL >= 8 ? 1 : 8 / NL); ++i) s.sy[r0 + k + at / 4][local + at % 4 + i] = ys[i];
                        at = spread_first<8, GROUPS>(lane / NL);
#pragma unroll
                        for (int i = 0; i < 8 / GROUPS; ++i) s.few[warp][r0 + k + at / 4][NP + n0 + at % 4 + i] = cs[i];
                    }
                }
#pragma unroll
                for (int k = 2; k >= 0; k -= 2) {
                    float bs[8];
#pragma unroll
                    for (int i = 1; i >= 0; --i) {
                        const int r = r0 + k + i;
                        pair32 d[2], u[2], v[2], s1[2] = {0, 0}, s2[2] = {0, 0};
                        pair32 b[NPT], cc[NPT];
                        load_pairs(&s.sd[r][local], d);
                        load_pairs(&s.su[r][local], u);
                        load_pairs(&s.sg[r][local], v);
                        load_few<NPT>(&s.sB[r][n0], b);
                        load_few<NPT>(&s.sC[r][n0], cc);
                        if (flag >> r & 1) {
#pragma unroll
                            for (int n = 0; n < NPT; ++n) g[n][0] = g[n][1] = 0;
                        }
#pragma unroll
                        for (int n = 0; n < NPT; ++n) {
                            pair32 sum = 0;
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                g[n][p] = fma2(cc[n], v[p], g[n][p]);
                                sum = fma2(g[n][p], u[p], sum);
                                s1[p] = fma2(g[n][p], b[n], s1[p]);
                                const pair32 qq = mul2(g[n][p], q[k + i][n][p]);
                                s2[p] = fma2(qq, A[n][p], s2[p]);
                                dA[n][p] = fma2(qq, d[p], dA[n][p]);
                                g[n][p] = mul2(g[n][p], f[k + i][n][p]);
                            }
                            const float2 e = parts(sum);
                            bs[4 * i + n] = e.x + e.y;
                        }
                        float both[8];
                        const float2 e = parts(s1[0]), o = parts(s1[1]), e2 = parts(s2[0]), o2 = parts(s2[1]);
                        both[0] = e.x, both[1] = e.y, both[2] = o.x, both[3] = o.y;
                        both[4] = e2.x, both[5] = e2.y, both[6] = o2.x, both[7] = o2.y;
                        // every lane of the channels has read this step's row: the sums take its place
                        spread_sum<8, NL, 1>(both, lane);
                        const int at = spread_first<8, NL>(ln);
                        float *to = (at < 4 ? &s.su[r][local] : &s.sg[r][local - 4]) + at;
#pragma unroll
                        for (int j = 0; j < (NL >= 8 ? 1 : 8 / NL); ++j) to[j] = both[j];
                    }
                    spread_sum<8, GROUPS, NL>(bs, lane);
                    const int at = spread_first<8, GROUPS>(lane / NL);
#pragma unroll
                    for (int i = 0; i < 8 / GROUPS; ++i) s.few[warp][r0 + k + at / 4][n0 + at % 4 + i] = bs[i];
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < kSteps * 2 * NP; i += kThreads) {
                const int r = i / (2 * NP), n = i % (2 * NP);
                if (r >= rows) break;
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < kThreads / 32; ++k) sum += s.few[k][r][n];
                const long long row = (long long)(t + r) * a.Be + w.e;
                a.few[(((long long)(tile - w.group * a.group_tiles) * a.T * a.Be + row) * a.groups + w.group) * (2 * NP) + n] = sum;
            }
            {
                R rx, rt, rg, rz;
                rx.fetch(x + t * sx, sx, rows, cols);
                rt.fetch(dt + t * st, st, rows, cols);
                rg.fetch(dy + t * sy, sy, rows, cols);
                if (z) rz.fetch(z + t * sz, sz, rows, cols);
                T *dx = static_cast<T *>(a.dx) + w.e * a.ldx + w.c0, *ddt = static_cast<T *>(a.ddt) + w.e * a.lddt + w.c0;
                T *dz = z ? static_cast<T *>(a.dz) + w.e * a.ldz + w.c0 : nullptr;
                float sumD[R::V] = {}, sumb[R::V] = {};
#pragma unroll
                for (int i = 0; i < R::PASSES; ++i) {
                    const int r = R::row(i), l = R::col(i);
                    if (r >= kSteps || r >= rows || l >= cols) continue;
                    float d[R::V], s1[R::V], s2[R::V], xv[R::V], tv[R::V], gv[R::V], D[R::V], bias[R::V], o[R::V];
                    get_floats(&s.sD[l], D);
                    get_floats(&s.sbias[l], bias);
                    get_floats(&s.sd[r][l], d);
                    get_floats(&s.su[r][l], s1);
                    get_floats(&s.sg[r][l], s2);
                    rx.get(i, xv);
                    rt.get(i, tv);
                    rg.get(i, gv);
                    if (z) {
                        float zv[R::V], yv[R::V];
                        rz.get(i, zv);
                        get_floats(&s.sy[r][l], yv);
#pragma unroll
                        for (int k = 0; k < R::V; ++k) {
                            const float p = sigmoid_fast(zv[k]), all = a.D ? fmaf(D[k], xv[k], yv[k]) : yv[k];
                            o[k] = gv[k] * all * (p * fmaf(zv[k], 1.f - p, 1.f));
                            gv[k] *= zv[k] * p;
                        }
                        R::put(dz + (t + r) * sz + l, o);
                    }
#pragma unroll
                    for (int k = 0; k < R::V; ++k) {
                        o[k] = a.D ? fmaf(d[k], s1[k], D[k] * gv[k]) : d[k] * s1[k];
                        sumD[k] = fmaf(gv[k], xv[k], sumD[k]);
                    }
                    R::put(dx + (t + r) * sx + l, o);
#pragma unroll
                    for (int k = 0; k < R::V; ++k) {
                        o[k] = fmaf(xv[k], s1[k], kLn2 * s2[k]);
                        if (a.softplus) o[k] *= sigmoid_fast(tv[k] + bias[k]);
                        sumb[k] += o[k];
                    }
                    R::put(ddt + (t + r) * st + l, o);
                }
#pragma unroll
                for (int k = 0; k < R::V; ++k) {
                    add_to(s.kept[0][0][k][threadIdx.x], s.kept[0][1][k][threadIdx.x], sumD[k]);
                    add_to(s.kept[1][0][k][threadIdx.x], s.kept[1][1][k][threadIdx.x], sumb[k]);
                }
            }
            float f[4][NPT];
            unpack<NPT>(dA, f);
#pragma unroll
            for (int n = 0; n < 16; ++n) add_to(s.dA[0][n][threadIdx.x], s.dA[1][n][threadIdx.x], f[n / 4][n % 4]);
#pragma unroll
            for (int n = 0; n < NPT; ++n) dA[n][0] = dA[n][1] = 0;
        }
        if (a.dstate_in && w.t0 == 0) {
            float f[4][NPT];
            unpack<NPT>(g, f);
            store_state<NPT>(a.dstate_in, a, w.e, c, w.c1, n0, f);
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)slice * a.channels * (a.N + 2);
    {
        float f[4][NPT];
#pragma unroll
        for (int n = 0; n < 16; ++n) f[n / 4][n % 4] = s.dA[0][n][threadIdx.x] + s.dA[1][n][threadIdx.x];
        store_state<NPT>(part, a, 0, c, w.c1, n0, f);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * CT; i += kThreads) {
        const int k = i / CT, l = i % CT;
        if (l >= cols) continue;
        float sum = 0.f;
        for (int r = 0; r < kThreads / R::COLS; ++r) {
            const int i = r * R::COLS + l / R::V;
            sum += s.kept[k][0][l % R::V][i] + s.kept[k][1][l % R::V][i];
        }
        part[(size_t)a.channels * (a.N + k) + w.c0 + l] = sum;
    }
}

// The gradients of B and C from the shares of a group's tiles.
template <typename T, int NP>
__global__ void __launch_bounds__(256) scan_few_kernel(ScanArgs a) {
    grid_wait();
    const long long all = (long long)a.T * a.Be * a.groups * 2 * NP, i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    float sum = 0.f;
#pragma unroll 8
    for (int k = 0; k < a.group_tiles; ++k) sum += a.few[k * all + i];
    const int n = (int)(i % NP), which = (int)(i / NP % 2);
    const long long at = i / (2 * NP), row = at / a.groups, group = at - row * a.groups;
    if (n >= a.N) return;
    if (which == 0) static_cast<T *>(a.dB)[row * a.ldb + group * a.N + n] = from_f32<T>(sum);
    else static_cast<T *>(a.dC)[row * a.ldc + group * a.N + n] = from_f32<T>(sum);
}

// One step, the state in place: NL lanes share a channel, four elements each.
template <typename T, int NL>
__global__ void __launch_bounds__(256) scan_step_kernel(ScanArgs a, int envs) {
    grid_wait();
    constexpr int CHANNELS = 256 / NL;
    const int cols = (a.channels + CHANNELS - 1) / CHANNELS, c = blockIdx.x % cols * CHANNELS + threadIdx.x / NL, n0 = threadIdx.x % NL * 4;
    const int e0 = blockIdx.x / cols * envs;
    const bool on = c < a.channels, whole = a.N % 4 == 0;
    float A[4] = {}, D = 0.f, bias = 0.f;
    const int group = on ? c / a.per : 0;
    if (on) {
#pragma unroll
        for (int n = 0; n < 4; ++n) A[n] = n0 + n < a.N ? a.A[(long long)c * a.N + n0 + n] * kLog2e : 0.f;
        if (a.D) D = a.D[c];
        if (a.bias) bias = a.bias[c];
    }
    for (int e = e0; e < min(a.Be, e0 + envs); ++e) {
        float h[4] = {}, y = 0.f, x = 0.f;
        float *state = a.state_out + ((long long)e * a.channels + c) * a.N + n0;
        if (on) {
            const bool empty = a.done && a.done[e];
            if (whole) {
                if (n0 < a.N && !empty) {
                    const float4 f = *reinterpret_cast<const float4 *>(state);
                    h[0] = f.x, h[1] = f.y, h[2] = f.z, h[3] = f.w;
                }
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (n0 + n < a.N && !empty) h[n] = state[n];
            }
            x = to_f32(static_cast<const T *>(a.x)[e * a.ldx + c]);
            float d = to_f32(static_cast<const T *>(a.dt)[e * a.lddt + c]) + bias;
            if (a.softplus) d = softplus_fast(d);
            const T *B = static_cast<const T *>(a.B) + e * a.ldb + (long long)group * a.N + n0, *C = static_cast<const T *>(a.C) + e * a.ldc + (long long)group * a.N + n0;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                if (n0 + n >= a.N) break;
                h[n] = fmaf(exp2_fast(d * A[n]), h[n], d * x * to_f32(B[n]));
                y = fmaf(to_f32(C[n]), h[n], y);
            }
            if (whole) {
                if (n0 < a.N) *reinterpret_cast<float4 *>(state) = make_float4(h[0], h[1], h[2], h[3]);
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (n0 + n < a.N) state[n] = h[n];
            }
        }
#pragma unroll
        for (int o = NL / 2; o > 0; o /= 2) y += __shfl_xor_sync(0xffffffffu, y, o);
        if (on && n0 == 0) {
            y = fmaf(D, x, y);
            if (a.z) {
                const float z = to_f32(static_cast<const T *>(a.z)[e * a.ldz + c]);
                y *= z * sigmoid_fast(z);
            }
            static_cast<T *>(a.y)[e * a.ldy + c] = from_f32<T>(y);
        }
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

// By sizes alone, so that the workspace and the order of sums go by them.
struct Plan {
    int NL, CT, NP, tiles, group_tiles, len, nseg, parts;
    size_t seg, sums, mark, few, part;  // floats of each area of the workspace
};
Plan plan_of(const ppo_selective_scan_desc *d, bool bwd) {
    Plan p = {};
    p.NL = d->N <= 16 ? 4 : d->N <= 32 ? 8 : 16;
    p.NP = 4 * p.NL;
    p.CT = 512 / p.NL;
    const auto up = [](size_t n) { return (n + 7) & ~(size_t)7; };  // whole 32 bytes
    p.group_tiles = ppo_cdiv(d->channels / d->groups, p.CT);
    p.tiles = p.group_tiles * d->groups;
    const long long blocks = (long long)d->Be * p.tiles, want = (bwd ? 2 : 4) * 148;
    long long n = blocks < want ? want / blocks : 1;
    const int most = ppo_cdiv(d->T, 64);
    if (n > most) n = most;
    p.len = ppo_cdiv(ppo_cdiv(d->T, n), kSteps) * kSteps;
    p.nseg = ppo_cdiv(d->T, p.len);
    const size_t held = (size_t)d->Be * p.tiles * kThreads * 16;
    if (p.nseg > 1) {
        p.seg = p.nseg * held;
        p.sums = up((size_t)p.nseg * d->Be * (d->channels + 1));
    }
    if (bwd) {
        p.mark = ppo_cdiv(d->T, 4) * held;
        p.few = (size_t)d->T * d->Be * p.tiles * 2 * p.NP;
        const long long items = (long long)d->Be * p.nseg, per = p.tiles < 2 * 148 ? 2 * 148 / p.tiles : 1;  // one round of two blocks an SM
        p.parts = (int)(items < per ? items : per);
        p.part = up((size_t)p.parts * d->channels * (d->N + 2));
    }
    return p;
}

ScanArgs args(const ppo_selective_scan_desc *d, const Plan &p, const void *x, const void *dt, const float *A, const void *B, const void *C,
              const float *D, const void *z, const float *bias) {
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
    a.per = d->channels / d->groups;
    a.softplus = d->softplus;
    a.tiles = p.tiles;
    a.group_tiles = p.group_tiles;
    a.len = p.len;
    a.nseg = p.nseg;
    a.parts = p.parts;
    return a;
}

// Rows of whole, aligned vectors of 16 bytes, also where a group ends.
bool vectors(const ppo_selective_scan_desc *d, std::initializer_list<const void *> ps) {
    const int V = 16 / (int)elem_bytes(d->dtype);
    return d->channels / d->groups % V == 0 && d->ldx % V == 0 && d->lddt % V == 0 && d->ldz % V == 0 && d->ldy % V == 0 && !misaligned(ps, 16);
}

// fn(T{}, lanes of a channel, whether rows are vectors)
template <typename F>
int with_shape(const ppo_selective_scan_desc *d, const Plan &p, bool vec, F &&fn) {
    return with_elem(d->dtype, [&](auto t) -> int {
        const auto lanes = [&](auto v) -> int {
            if (p.NL == 4) return fn(t, std::integral_constant<int, 4>{}, v);
            if (p.NL == 8) return fn(t, std::integral_constant<int, 8>{}, v);
            return fn(t, std::integral_constant<int, 16>{}, v);
        };
        return vec ? lanes(std::true_type{}) : lanes(std::false_type{});
    });
}

}  // namespace

extern "C" size_t ppo_selective_scan_workspace_bytes(const ppo_selective_scan_desc *d, int backward) {
    if (check(d) != PPO_OK) return 0;
    const Plan p = plan_of(d, backward != 0);
    return ((backward ? 2 : 1) * p.seg + p.sums + p.mark + p.few + p.part) * sizeof(float);
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
    const Plan p = plan_of(d, false);
    ScanArgs a = args(d, p, x, dt, A, B, C, D, z, dt_bias);
    a.done = done;
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    a.seg = static_cast<float *>(workspace);
    a.sum = a.seg + p.seg;
    a.cut = reinterpret_cast<int *>(a.sum + (size_t)p.nseg * d->Be * d->channels);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned blocks = (unsigned)(d->Be * p.tiles);
    return with_shape(d, p, vectors(d, {x, dt, z, y}), [&](auto t, auto nl, auto v) -> int {
        using T = decltype(t);
        constexpr int NL = decltype(nl)::value;
        constexpr bool VEC = decltype(v)::value;
        // the last segment hands nothing on
        if (p.nseg > 1) PPO_TRY(ppo_launch(scan_kernel<T, 4, NL, ENDS, VEC>, dim3(blocks * (p.nseg - 1)), dim3(kThreads), 0, st, a));
        return ppo_launch(scan_kernel<T, 4, NL, OUTPUT, VEC>, dim3(blocks * p.nseg), dim3(kThreads), 0, st, a);
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
    const Plan p = plan_of(d, true);
    ScanArgs a = args(d, p, x, dt, A, B, C, D, z, dt_bias);
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
    a.seg = static_cast<float *>(workspace);
    a.back = a.seg + p.seg;
    a.mark = a.back + p.seg;
    a.few = a.mark + p.mark;
    const bool params = dA || dD || ddt_bias;
    a.part = params ? a.few + p.few : nullptr;
    a.sum = a.few + p.few + p.part;
    a.cut = reinterpret_cast<int *>(a.sum + (size_t)p.nseg * d->Be * d->channels);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const unsigned blocks = (unsigned)(d->Be * p.tiles) * p.nseg;
    PPO_TRY(with_shape(d, p, vectors(d, {x, dt, z, dy, dx, ddt, dz}), [&](auto t, auto nl, auto v) -> int {
        using T = decltype(t);
        constexpr int NL = decltype(nl)::value;
        constexpr bool VEC = decltype(v)::value;
        constexpr size_t smem = sizeof(GradShared<T, NL, VEC>);
        static PerDevice<bool> allowed;
        PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(scan_bwd_kernel<T, NL, VEC>, smem); }));
        if (p.nseg > 1) PPO_TRY(ppo_launch(scan_kernel<T, 4, NL, BOTH, VEC>, dim3(blocks), dim3(kThreads), 0, st, a));
        PPO_TRY(ppo_launch(scan_kernel<T, 4, NL, MARKS, VEC>, dim3(blocks), dim3(kThreads), 0, st, a));
        PPO_TRY(ppo_launch(scan_bwd_kernel<T, NL, VEC>, dim3((unsigned)(p.tiles * p.parts)), dim3(kThreads), smem, st, a));
        const long long few = (long long)d->T * d->Be * d->groups * 2 * p.NP;
        return ppo_launch(scan_few_kernel<T, 4 * NL>, dim3((unsigned)((few + 255) / 256)), dim3(256), 0, st, a);
    }));
    return params ? ppo_param_sum(a.part, p.parts, {{dA, dD, ddt_bias}, {d->channels * d->N, d->channels, d->channels}}, accumulate, st) : PPO_OK;
}

extern "C" int ppo_selective_scan_step(const ppo_selective_scan_desc *d, const void *x, const void *dt, const float *A, const void *B, const void *C,
                                       const float *D, const void *z, const float *dt_bias, const uint8_t *start, float *state, void *y, void *stream) {
    PPO_TRY(check(d));
    if (d->T != 1) return PPO_ERR_SHAPE;
    if (!x || !dt || !A || !B || !C || !state || !y) return PPO_ERR_INVALID_ARG;
    if (misaligned({x, dt, B, C, z, y}, elem_bytes(d->dtype)) || misaligned({A, D, dt_bias}, 4) || misaligned({state}, 16)) return PPO_ERR_ALIGN;
    ScanArgs a = args(d, {}, x, dt, A, B, C, D, z, dt_bias);
    a.done = start;
    a.y = y;
    a.state_out = state;
    return with_elem(d->dtype, [&](auto t) -> int {
        using T = decltype(t);
        const auto run = [&](auto nl) -> int {
            constexpr int NL = decltype(nl)::value;
            const long long cols = ppo_cdiv(d->channels, 256 / NL);
            int envs = (int)(cols * d->Be / (8 * 148));  // as many envs a block as leave every SM eight
            if (envs < 1) envs = 1;
            return ppo_launch(scan_step_kernel<T, NL>, dim3((unsigned)(cols * ppo_cdiv(d->Be, envs))), dim3(256), 0, static_cast<cudaStream_t>(stream), a, envs);
        };
        if (d->N <= 4) return run(std::integral_constant<int, 1>{});
        if (d->N <= 8) return run(std::integral_constant<int, 2>{});
        if (d->N <= 16) return run(std::integral_constant<int, 4>{});
        if (d->N <= 32) return run(std::integral_constant<int, 8>{});
        return run(std::integral_constant<int, 16>{});
    });
}
