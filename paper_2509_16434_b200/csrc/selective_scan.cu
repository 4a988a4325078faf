// Selective scan: states whose decay and input the data choose, and its gradients.
//
// h_t = exp(d_t A) h_{t-1} + d_t x_t B_t: one exponential and four multiply-adds for each element of a state and step, against 8 bytes
// for each channel and step in 16 bits: with 16 elements a channel the exponentials (16 a clock and SM) bound it, not memory.
//
// Forwards a thread takes a channel, or two neighbouring ones, of one env through the steps, with 16 elements of the states in registers (channels
// with more of them belong to two or four lanes): nothing is shared but the rows of B and C, and a step's sum over the elements is the
// thread's own.  Backwards four channels by four elements are a thread's, since there sums go over the channels as well as over the elements.
// States, sums and arithmetic in 32 bits, packed arithmetic on two numbers at a time.
//
// Long sequences of few channels are cut into segments: a pass makes what each segment ends with, and each starts from the ends in front of it.
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
    // Of every segment and env, [channels][NP] (N padded): the states it ends with (starting from zeros, but for the first one; in the last one's place
    // the state that comes in) and the gradients it hands to the steps in front (getting zeros; in the first one's place the gradient
    // of the state that is left); what its step sizes add up to for each channel, and whether a flag is set in it.
    float *seg, *back, *sum;
    int *cut;
    float *mark;  // the states in front of every fourth step, [ceil(T / 4)][Be][channels][NP]
    float *few;   // shares of the gradients of B and C, [group_tiles][T * Be][groups][2][NP]
    float *part;  // shares of the gradients of A, D and dt_bias, [parts][channels * (N + 2)]
    int parts;
};

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

// Backwards NL lanes share four channels and hold four elements each of their states.
template <int NL>
struct Shape {
    static constexpr int NP = 4 * NL, GROUPS = 32 / NL, CT = 4 * GROUPS * (kThreads / 32);
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

// Elements n0 .. n0 + W - 1 of a state of N in memory; zeros behind the last one.
template <int W>
__device__ __forceinline__ void load_row(const float *p, int N, int n0, float (&h)[W]) {
    const bool whole = N % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
#pragma unroll
    for (int n = 0; n < W; n += 4) {
        if (whole) {
            const float4 f = n0 + n < N ? *reinterpret_cast<const float4 *>(p + n0 + n) : make_float4(0.f, 0.f, 0.f, 0.f);
            h[n] = f.x, h[n + 1] = f.y, h[n + 2] = f.z, h[n + 3] = f.w;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) h[n + i] = n0 + n + i < N ? p[n0 + n + i] : 0.f;
        }
    }
}
template <int W>
__device__ __forceinline__ void store_row(float *p, int N, int n0, const float (&h)[W]) {
    const bool whole = N % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
#pragma unroll
    for (int n = 0; n < W; n += 4) {
        if (whole) {
            if (n0 + n < N) *reinterpret_cast<float4 *>(p + n0 + n) = make_float4(h[n], h[n + 1], h[n + 2], h[n + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + n + i < N) p[n0 + n + i] = h[n + i];
        }
    }
}
__device__ __forceinline__ void load_pairs(const float *p, pair32 (&v)[2]) {
    const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p);
    v[0] = u.x, v[1] = u.y;
}
__device__ __forceinline__ void load_few(const float2 *p, pair32 (&v)[4]) {
#pragma unroll
    for (int n = 0; n < 4; n += 2) {
        const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p + n);
        v[n] = u.x, v[n + 1] = u.y;
    }
}

// Takes elements n0 .. of a channel's state, or gradient, through segment s: exp2(A sum of its step sizes) h + add, or add alone behind a flag.  from: what
// each segment adds; A: times log2(e).
template <int W>
__device__ __forceinline__ void through(const ScanArgs &a, int NP, int s, int e, int c, int n0, const float (&A)[W], const float *from, float (&h)[W]) {
    const long long at = (long long)s * a.Be + e;
    float add[W];
    load_row<W>(from + (at * a.channels + c) * NP, NP, n0, add);
    const bool cut = a.cut[at];
    const float d = a.sum[at * a.channels + c];
#pragma unroll
    for (int n = 0; n < W; ++n) h[n] = cut ? add[n] : fmaf(exp2_fast(d * A[n]), h[n], add[n]);
}
// What a segment starts from: the state that comes in, or what the first segment ends with, taken through the segments in between.
template <int W>
__device__ __forceinline__ void start_of(const ScanArgs &a, int NP, const Work &w, int c, int n0, const float (&A)[W], float (&h)[W]) {
    const long long at = (long long)(w.seg == 0 ? a.nseg - 1 : 0) * a.Be + w.e;
    load_row<W>(a.seg + (at * a.channels + c) * NP, NP, n0, h);
    for (int s = 1; s < w.seg; ++s) through<W>(a, NP, s, w.e, c, n0, A, a.seg, h);
}
// The gradient that a segment gets of the state it leaves.
template <int W>
__device__ __forceinline__ void end_of(const ScanArgs &a, int NP, const Work &w, int c, int n0, const float (&A)[W], float (&g)[W]) {
    load_row<W>(a.back + ((long long)w.e * a.channels + c) * NP, NP, n0, g);
    for (int s = a.nseg - 1; s > w.seg; --s) through<W>(a, NP, s, w.e, c, n0, A, a.back, g);
}

enum Mode {
    OUTPUT,  // y and the state that is left
    ENDS,    // what each segment ends with
    BOTH,    // that, and the gradients it hands to the steps in front
    MARKS    // the states in front of every fourth step
};

// CPT neighbouring channels of a row, as they lie in memory.
template <typename T, int CPT>
struct Cell {
    using Word = std::conditional_t<CPT == 1, T, std::conditional_t<sizeof(T) == 2, uint32_t, uint2>>;
    Word w;
    __device__ __forceinline__ void load(const T *p) { w = *reinterpret_cast<const Word *>(p); }
    // the second one of a single channel is 0
    __device__ __forceinline__ pair32 get() const {
        if constexpr (CPT == 1) {
            return pair_of(to_f32(w), 0.f);
        } else {
            Vec<T> v;
            float f[Vec<T>::N];
            if constexpr (sizeof(T) == 2) v.raw = make_uint4(w, 0, 0, 0);
            else v.raw = make_uint4(w.x, w.y, 0, 0);
            v.get(f);
            return pair_of(f[0], f[1]);
        }
    }
    static __device__ __forceinline__ pair32 softplus(pair32 v) {
        if constexpr (CPT == 1) return pair_of(softplus_fast(parts(v).x), 0.f);
        else return softplus_pair(v);
    }
    static __device__ __forceinline__ pair32 silu(pair32 v) {
        if constexpr (CPT == 1) return pair_of(parts(v).x * sigmoid_fast(parts(v).x), 0.f);
        else return mul2(v, sigmoid_pair(v));
    }
    static __device__ __forceinline__ void put(T *p, pair32 v) {
        const float2 f = parts(v);
        if constexpr (CPT == 1) {
            *p = from_f32<T>(f.x);
        } else {
            float all[Vec<T>::N] = {f.x, f.y};
            Vec<T> r;
            r.set(all);
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t *>(p) = r.raw.x;
            else *reinterpret_cast<uint2 *>(p) = make_uint2(r.raw.x, r.raw.y);
        }
    }
};

// The rows of B and C of kSteps steps on their way from memory to shared memory, padded with zeros.
template <typename T, int NP, bool WITH_C>
struct FewRows {
    static constexpr int EACH = kSteps * NP / kThreads;
    static_assert(kThreads % NP == 0);
    T b[EACH], c[WITH_C ? EACH : 1];
    // B, C: of the first step
    __device__ __forceinline__ void fetch(const T *B, const T *C, long long sb, long long sc, int rows, int N) {
        const int n = threadIdx.x % NP, t0 = threadIdx.x / NP;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int t = t0 + i * (kThreads / NP);
            const bool ok = t < rows && n < N;
            b[i] = ok ? B[t * sb + n] : from_f32<T>(0.f);
            if (WITH_C) c[i] = ok ? C[t * sc + n] : from_f32<T>(0.f);
        }
    }
    __device__ __forceinline__ void put(float (&B)[kSteps][NP], float (&C)[WITH_C ? kSteps : 1][NP]) const {
        const int n = threadIdx.x % NP, t0 = threadIdx.x / NP;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            B[t0 + i * (kThreads / NP)][n] = to_f32(b[i]);
            if (WITH_C) C[t0 + i * (kThreads / NP)][n] = to_f32(c[i]);
        }
    }
};

template <typename T, int NL, int CPT, int MODE>
__global__ void __launch_bounds__(kThreads, CPT == 2 && MODE == OUTPUT ? 3 : 4) scan_kernel(ScanArgs a) {
    grid_wait();
    constexpr int W = 16, P = W / 2, NP = W * NL, CT = kThreads / NL * CPT;
    constexpr bool WITH_C = MODE == OUTPUT || MODE == BOTH, WITH_DY = MODE == BOTH, WITH_Z = MODE == OUTPUT || MODE == BOTH;
    using Word = Cell<T, CPT>;
    __shared__ alignas(16) float sB[2][kSteps][NP], sC[2][WITH_C ? kSteps : 1][NP];
    const Work w = work_of<CT>(a, blockIdx.x % a.tiles, blockIdx.x / a.tiles);
    const int ln = threadIdx.x % NL, c = w.c0 + threadIdx.x / NL * CPT, n0 = ln * W;
    const bool on = c < w.c1;
    const long long sx = a.Be * a.ldx, st = a.Be * a.lddt, sb = a.Be * a.ldb, sc = a.Be * a.ldc, sz = a.Be * a.ldz, sy = a.Be * a.ldy;
    const T *x = static_cast<const T *>(a.x) + w.e * a.ldx + c + w.t0 * sx, *dt = static_cast<const T *>(a.dt) + w.e * a.lddt + c + w.t0 * st;
    const T *B = static_cast<const T *>(a.B) + w.e * a.ldb + (long long)w.group * a.N + w.t0 * sb;
    const T *C = static_cast<const T *>(a.C) + w.e * a.ldc + (long long)w.group * a.N + w.t0 * sc;
    const T *z = WITH_Z && a.z ? static_cast<const T *>(a.z) + w.e * a.ldz + c + w.t0 * sz : nullptr;
    const T *dy = WITH_DY ? static_cast<const T *>(a.dy) + w.e * a.ldy + c + w.t0 * sy : nullptr;
    T *y = MODE == OUTPUT ? static_cast<T *>(a.y) + w.e * a.ldy + c + w.t0 * sy : nullptr;

    Word rx[4], rt[4], rz[WITH_Z ? 4 : 1], rg[WITH_DY ? 4 : 1];
    const auto fetch = [&](int rows) {  // of the four steps at x, dt, z and dy
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!on || k >= rows) break;
            rx[k].load(x + k * sx);
            rt[k].load(dt + k * st);
            if (WITH_Z && z) rz[k].load(z + k * sz);
            if (WITH_DY) rg[k].load(dy + k * sy);
        }
    };
    fetch(w.t1 - w.t0);
    FewRows<T, NP, WITH_C> few;
    few.fetch(B, C, sb, sc, w.t1 - w.t0, a.N);

    pair32 A[CPT][P], h[CPT][P], Pr[WITH_DY ? P : 1], G[WITH_DY ? P : 1], D = 0, bias = 0;
    const long long held = ((long long)w.seg * a.Be + w.e) * a.channels;
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
        float Af[W] = {}, f[W] = {};
        if (on) {
            load_row<W>(a.A + (long long)(c + j) * a.N, a.N, n0, Af);
#pragma unroll
            for (int n = 0; n < W; ++n) Af[n] *= kLog2e;
            if (MODE == ENDS || MODE == BOTH || a.nseg == 1) {
                if (w.seg == 0) {
                    if (a.state_in) load_row<W>(a.state_in + ((long long)w.e * a.channels + c + j) * a.N, a.N, n0, f);
                    if (a.nseg > 1) store_row<W>(a.seg + (held + (long long)(a.nseg - 1) * a.Be * a.channels + c + j) * NP, NP, n0, f);
                }
            } else {
                start_of<W>(a, NP, w, c + j, n0, Af, f);
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            A[j][i] = pair_of(Af[2 * i], Af[2 * i + 1]);
            h[j][i] = pair_of(f[2 * i], f[2 * i + 1]);
        }
    }
    if (on) {
        if (a.D && MODE == OUTPUT) D = pair_of(a.D[c], CPT == 2 ? a.D[c + CPT - 1] : 0.f);
        if (a.bias) bias = pair_of(a.bias[c], CPT == 2 ? a.bias[c + CPT - 1] : 0.f);
    }
    if constexpr (WITH_DY) {
#pragma unroll
        for (int i = 0; i < P; ++i) Pr[i] = twice(1.f), G[i] = 0;
    }
    few.put(sB[0], sC[0]);
    __syncthreads();
    pair32 total = 0;
    bool cut = false;
    int buffer = 0;
    for (int t = w.t0; t < w.t1; t += kSteps, buffer ^= 1) {
        const int rows = w.t1 - t;
        const uint32_t flag = flags_of(a, w.e, t, rows);
        B += kSteps * sb;
        C += kSteps * sc;
        if (rows > kSteps) few.fetch(B, C, sb, sc, rows - kSteps, a.N);
#pragma unroll 1
        for (int s = 0; s < kSteps && s < rows; s += 4) {
            if constexpr (MODE == MARKS) {
                float *to = a.mark + (((long long)((t + s) / 4) * a.Be + w.e) * a.channels + c) * NP + n0;
#pragma unroll
                for (int j = 0; j < CPT; ++j)
#pragma unroll
                    for (int i = 0; i < P; i += 2)
                        if (on) *reinterpret_cast<ulonglong2 *>(to + j * NP + 2 * i) = make_ulonglong2(h[j][i], h[j][i + 1]);
            }
            pair32 xs[4], ds[4], zs[4], gs[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                xs[k] = ds[k] = zs[k] = gs[k] = 0;
                if (!on || s + k >= rows) continue;
                xs[k] = rx[k].get();
                ds[k] = add2(rt[k].get(), bias);
                if (a.softplus) ds[k] = Word::softplus(ds[k]);
                if (WITH_Z && z) zs[k] = Word::silu(rz[k].get());
                if (WITH_DY) gs[k] = rg[k].get();
                if (WITH_DY && z) gs[k] = mul2(gs[k], zs[k]);
            }
            x += 4 * sx;
            dt += 4 * st;
            if (WITH_Z && z) z += 4 * sz;
            if (WITH_DY) dy += 4 * sy;
            fetch(rows - s - 4);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                pair32 out[CPT];
                const float2 d = parts(ds[k]), u = parts(mul2(ds[k], xs[k])), g = parts(gs[k]);
#pragma unroll
                for (int j = 0; j < CPT; ++j) out[j] = 0;
#pragma unroll
                for (int i = 0; i < P; i += 2) {
                    pair32 b[2], cc[2] = {};
                    load_pairs(&sB[buffer][s + k][n0 + 2 * i], b);
                    if constexpr (WITH_C) load_pairs(&sC[buffer][s + k][n0 + 2 * i], cc);
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int j = 0; j < CPT; ++j) {
                            const pair32 f = exp2_pair(mul2(twice(j == 0 ? d.x : d.y), A[j][i + m]));
                            h[j][i + m] = fma2(f, h[j][i + m], mul2(twice(j == 0 ? u.x : u.y), b[m]));
                            if constexpr (MODE == OUTPUT) out[j] = fma2(cc[m], h[j][i + m], out[j]);
                            if constexpr (WITH_DY) {
                                Pr[i + m] = mul2(Pr[i + m], f);
                                if (!cut) G[i + m] = fma2(mul2(Pr[i + m], twice(g.x)), cc[m], G[i + m]);
                            }
                        }
                }
                if constexpr (MODE == ENDS || MODE == BOTH) total = add2(total, ds[k]);
                if constexpr (MODE == OUTPUT) {
                    const float2 o = parts(out[0]), q = parts(out[CPT - 1]);
                    float lo = o.x + o.y, hi = CPT == 2 ? q.x + q.y : 0.f;
#pragma unroll
                    for (int m = NL / 2; m > 0; m /= 2) {
                        lo += __shfl_xor_sync(0xffffffffu, lo, m);
                        if (CPT == 2) hi += __shfl_xor_sync(0xffffffffu, hi, m);
                    }
                    pair32 v = a.D ? fma2(D, xs[k], pair_of(lo, hi)) : pair_of(lo, hi);
                    if (z) v = mul2(v, zs[k]);
                    if (on && ln == 0 && s + k < rows) Word::put(y + k * sy, v);
                }
                if (flag >> (s + k) & 1) {
                    cut = true;
#pragma unroll
                    for (int j = 0; j < CPT; ++j)
#pragma unroll
                        for (int i = 0; i < P; ++i) h[j][i] = 0;
                }
            }
            if (MODE == OUTPUT) y += 4 * sy;
        }
        if (rows > kSteps) few.put(sB[buffer ^ 1], sC[buffer ^ 1]);
        __syncthreads();
    }
    if (!on) return;
    const long long at = (long long)w.seg * a.Be + w.e;
#pragma unroll
    for (int j = 0; j < CPT; ++j) {
        float f[W];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const float2 v = parts(h[j][i]);
            f[2 * i] = v.x, f[2 * i + 1] = v.y;
        }
        if constexpr (MODE == OUTPUT) {
            if (a.state_out && w.t1 == a.T) store_row<W>(a.state_out + ((long long)w.e * a.channels + c + j) * a.N, a.N, n0, f);
        }
        if constexpr (MODE == ENDS || MODE == BOTH) {
            if (w.seg < a.nseg - 1) store_row<W>(a.seg + (held + c + j) * NP, NP, n0, f);
            const float2 sums = parts(total);
            if (ln == 0) a.sum[at * a.channels + c + j] = j == 0 ? sums.x : sums.y;
        }
        if constexpr (MODE == BOTH) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 v = parts(G[i]);
                f[2 * i] = w.seg > 0 ? v.x : 0.f, f[2 * i + 1] = w.seg > 0 ? v.y : 0.f;
            }
            if (w.seg == 0 && a.dstate_out) load_row<W>(a.dstate_out + ((long long)w.e * a.channels + c + j) * a.N, a.N, n0, f);
            store_row<W>(a.back + (held + c + j) * NP, NP, n0, f);
        }
    }
    if constexpr (MODE == ENDS || MODE == BOTH) {
        if (threadIdx.x == 0 && w.tile == 0) a.cut[at] = cut;
    }
}

// Gradients.  Per step, with g = dL/dh_t and dv = dL/dy silu(z):
//   g_t = C_t dv_t + (nothing where done[t] is set, else) exp(d_{t+1} A) g_{t+1},   q = g_t exp(d_t A) h'_{t-1}
//   dC = sum_c dv h,  dB = sum_c g d x,  dx = D dv + d sum_n g B,  dd = x sum_n g B + sum_n q A,  dA += q d
// Four steps at a time, backwards: from the states in front of them forwards once more, which leaves the factors and exp(d A) h' of the
// four steps in registers (and y and the sums of dC on the way), then backwards over these.  A block goes through as many envs, or
// segments, as fall to it and keeps its shares of the parameters' gradients.
// Four elements of the states of four channels, [e][channel][N] in memory; zeros where there are none.
__device__ __forceinline__ void load_block(const float *from, const ScanArgs &a, int e, int c, int c1, int n0, float (&h)[4][4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int n = 0; n < 4; ++n) h[j][n] = 0.f;
        if (from && c + j < c1) load_row<4>(from + ((long long)e * a.channels + c + j) * a.N, a.N, n0, h[j]);
    }
}
__device__ __forceinline__ void store_block(float *to, const ScanArgs &a, int e, int c, int c1, int n0, const float (&h)[4][4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < c1) store_row<4>(to + ((long long)e * a.channels + c + j) * a.N, a.N, n0, h[j]);
}
// As pairs of neighbouring channels.
__device__ __forceinline__ void pack(const float (&h)[4][4], pair32 (&p)[4][2]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) p[n][0] = pair_of(h[0][n], h[1][n]), p[n][1] = pair_of(h[2][n], h[3][n]);
}
__device__ __forceinline__ void unpack(const pair32 (&p)[4][2], float (&h)[4][4]) {
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const float2 u = parts(p[n][0]), v = parts(p[n][1]);
        h[0][n] = u.x, h[1][n] = u.y, h[2][n] = v.x, h[3][n] = v.y;
    }
}

// A long sum as two numbers: what hi rounds away stays in lo (Knuth's error of a sum).
__device__ __forceinline__ void add_to(float &hi, float &lo, float v) {
    const float sum = __fadd_rn(hi, v), w = __fsub_rn(sum, hi);
    lo += __fadd_rn(__fsub_rn(hi, __fsub_rn(sum, w)), __fsub_rn(v, w));
    hi = sum;
}

template <typename T, int NL, bool VEC>
struct GradShared {
    static constexpr int CT = Shape<NL>::CT, NP = Shape<NL>::NP;
    float sd[kSteps][CT], su[kSteps][CT], sg[kSteps][CT], sy[kSteps][CT], sD[CT], sbias[CT];
    float2 sB[kSteps][NP], sC[kSteps][NP];
    float few[kThreads / 32][kSteps][2 * NP];
    float mark[4][4][kThreads * 4];
    float dA[2][16][kThreads], kept[2][2][Rows<T, CT, VEC>::V][kThreads];  // [..][2]: hi and lo of the sums
};

// Four numbers, or zeros.
__device__ __forceinline__ void copy_async(float *to, const float *from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

template <typename T, int NL, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) scan_bwd_kernel(ScanArgs a) {
    grid_wait();
    constexpr int NPT = 4;
    using S = Shape<NL>;
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
        load_block(a.A, a, 0, c, w.c1, n0, f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NPT; ++n) f[j][n] *= kLog2e;
        pack(f, A);
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
                load_block(a.dstate_out, a, w.e, c, w.c1, n0, f);
            } else {
                unpack(A, Af);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int n = 0; n < 4; ++n) f[j][n] = 0.f;
                    if (c + j < w.c1) end_of<4>(a, NP, w, c + j, n0, Af[j], f[j]);
                }
            }
            pack(f, g);
        }
        for (int t = w.t0 + (w.t1 - 1 - w.t0) / kSteps * kSteps; t >= w.t0; t -= kSteps) {
            const int rows = w.t1 - t;
            const uint32_t flag = flags_of(a, w.e, t, rows);
            __syncthreads();  // the tile behind is done with
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                if (4 * m >= rows) break;
                const float *from = a.mark + (((long long)(t / 4 + m) * a.Be + w.e) * a.channels + c) * NP + n0;
#pragma unroll
                for (int j = 0; j < 4; ++j) copy_async(&s.mark[m][j][threadIdx.x * 4], c + j < w.c1 ? from + j * NP : a.mark, c + j < w.c1);
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
                    float d[R::V], u[R::V], v[R::V];
                    if (r < rows && l < cols) {
                        rt.get(i, d);
                        rx.get(i, u);
                        rg.get(i, v);
                        float b[R::V], f[R::V];
                        get_floats(&s.sbias[l], b);
                        if (z) rz.get(i, f);
#pragma unroll
                        for (int k = 0; k < R::V; k += 2) {
                            constexpr int TWO = R::V > 1;
                            pair32 step = add2(pair_of(d[k], d[k + TWO]), pair_of(b[k], b[k + TWO]));
                            if (a.softplus) step = softplus_pair(step);
                            const float2 p = parts(step), q = parts(mul2(pair_of(u[k], u[k + TWO]), step));
                            d[k] = p.x, d[k + TWO] = p.y, u[k] = q.x, u[k + TWO] = q.y;
                            if (z) {
                                const pair32 zz = pair_of(f[k], f[k + TWO]);
                                const float2 g = parts(mul2(pair_of(v[k], v[k + TWO]), mul2(zz, sigmoid_pair(zz))));
                                v[k] = g.x, v[k + TWO] = g.y;
                            }
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < R::V; ++k) d[k] = u[k] = v[k] = 0.f;
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
                    float start[4][NPT];
#pragma unroll
                    for (int j = 0; j < 4; ++j) get_floats(&s.mark[m][j][threadIdx.x * 4], start[j]);
                    pack(start, h);
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
                            load_few(&s.sB[r][n0], b);
                            load_few(&s.sC[r][n0], cc);
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
                        load_few(&s.sB[r][n0], b);
                        load_few(&s.sC[r][n0], cc);
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
            unpack(dA, f);
#pragma unroll
            for (int n = 0; n < 16; ++n) add_to(s.dA[0][n][threadIdx.x], s.dA[1][n][threadIdx.x], f[n / 4][n % 4]);
#pragma unroll
            for (int n = 0; n < NPT; ++n) dA[n][0] = dA[n][1] = 0;
        }
        if (a.dstate_in && w.t0 == 0) {
            float f[4][NPT];
            unpack(g, f);
            store_block(a.dstate_in, a, w.e, c, w.c1, n0, f);
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)slice * a.channels * (a.N + 2);
    {
        float f[4][NPT];
#pragma unroll
        for (int n = 0; n < 16; ++n) f[n / 4][n % 4] = s.dA[0][n][threadIdx.x] + s.dA[1][n][threadIdx.x];
        store_block(part, a, 0, c, w.c1, n0, f);
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
    int NL, NP, len, nseg, parts;  // NL: lanes of a channel forwards
    int tiles, group_tiles;        // backwards
    size_t seg, sums, mark, few, part;  // floats of each area of the workspace
};
Plan plan_of(const ppo_selective_scan_desc *d, bool bwd) {
    Plan p = {};
    p.NL = d->N <= 16 ? 1 : d->N <= 32 ? 2 : 4;
    p.NP = 16 * p.NL;
    const auto up = [](size_t n) { return (n + 7) & ~(size_t)7; };  // whole 32 bytes
    const int per = d->channels / d->groups;
    p.group_tiles = ppo_cdiv(per, 128 / p.NL);
    p.tiles = p.group_tiles * d->groups;
    // segments: as many as give the GPU the warps that it can hold at a time, none shorter than 64 steps
    const long long warps = bwd ? 4ll * d->Be * p.tiles : (long long)d->Be * d->groups * ppo_cdiv(per, 64 / p.NL), want = (bwd ? 8 : 16) * 148;
    long long n = warps < want ? want / warps : 1;
    const int most = ppo_cdiv(d->T, 64);
    if (n > most) n = most;
    p.len = ppo_cdiv(ppo_cdiv(d->T, n), kSteps) * kSteps;
    p.nseg = ppo_cdiv(d->T, p.len);
    const size_t held = (size_t)d->Be * d->channels * p.NP;
    if (p.nseg > 1) {
        p.seg = p.nseg * held;
        p.sums = up((size_t)p.nseg * d->Be * (d->channels + 1));
    }
    if (bwd) {
        p.mark = ppo_cdiv(d->T, 4) * held;
        p.few = (size_t)d->T * d->Be * p.tiles * 2 * p.NP;
        const long long items = (long long)d->Be * p.nseg, slices = p.tiles < 2 * 148 ? 2 * 148 / p.tiles : 1;  // one round of two blocks an SM
        p.parts = (int)(items < slices ? items : slices);
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

// Rows of whole vectors of V elements, aligned to these, also where a group ends.
bool vectors(const ppo_selective_scan_desc *d, int V, std::initializer_list<const void *> ps) {
    return d->channels / d->groups % V == 0 && d->ldx % V == 0 && d->lddt % V == 0 && d->ldz % V == 0 && d->ldy % V == 0 &&
           !misaligned(ps, V * elem_bytes(d->dtype));
}

// fn(T{}, NL)
template <typename F>
int with_lanes(const ppo_selective_scan_desc *d, const Plan &p, F &&fn) {
    return with_elem(d->dtype, [&](auto t) -> int {
        if (p.NL == 1) return fn(t, std::integral_constant<int, 1>{});
        if (p.NL == 2) return fn(t, std::integral_constant<int, 2>{});
        return fn(t, std::integral_constant<int, 4>{});
    });
}
// A pass over the first `segs` segments, `two` channels a thread.
template <typename T, int NL, int CPT, int MODE>
int pass_of(ScanArgs a, int segs, cudaStream_t st) {
    a.group_tiles = ppo_cdiv(a.per, kThreads / NL * CPT);
    a.tiles = a.group_tiles * a.groups;
    return ppo_launch(scan_kernel<T, NL, CPT, MODE>, dim3((unsigned)(a.Be * a.tiles) * segs), dim3(kThreads), 0, st, a);
}
template <typename T, int NL, bool VEC>
int back_launch(const ScanArgs &a, cudaStream_t st) {
    constexpr size_t smem = sizeof(GradShared<T, NL, VEC>);
    static PerDevice<bool> allowed;
    PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(scan_bwd_kernel<T, NL, VEC>, smem); }));
    return ppo_launch(scan_bwd_kernel<T, NL, VEC>, dim3((unsigned)(a.tiles * a.parts)), dim3(kThreads), smem, st, a);
}
template <typename T, int NL, int MODE>
int pass(const ScanArgs &a, bool two, int segs, cudaStream_t st) {
    return two ? pass_of<T, NL, 2, MODE>(a, segs, st) : pass_of<T, NL, 1, MODE>(a, segs, st);
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
    const bool two = vectors(d, 2, {x, dt, z, y});
    return with_lanes(d, p, [&](auto t, auto nl) -> int {
        using T = decltype(t);
        constexpr int NL = decltype(nl)::value;
        if (p.nseg > 1) PPO_TRY((pass<T, NL, ENDS>(a, two, p.nseg - 1, st)));  // the last segment hands nothing on
        return pass<T, NL, OUTPUT>(a, two, p.nseg, st);
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
    const bool two = vectors(d, 2, {x, dt}), vec = vectors(d, 16 / (int)elem_bytes(d->dtype), {x, dt, z, dy, dx, ddt, dz});
    PPO_TRY(with_lanes(d, p, [&](auto t, auto nl) -> int {
        using T = decltype(t);
        constexpr int NL = decltype(nl)::value;
        if (p.nseg > 1) PPO_TRY((pass_of<T, NL, 1, BOTH>(a, p.nseg, st)));
        PPO_TRY((pass<T, NL, MARKS>(a, two, p.nseg, st)));
        PPO_TRY((vec ? back_launch<T, 4 * NL, true>(a, st) : back_launch<T, 4 * NL, false>(a, st)));
        const long long few = (long long)d->T * d->Be * d->groups * 2 * p.NP;
        return ppo_launch(scan_few_kernel<T, 16 * NL>, dim3((unsigned)((few + 255) / 256)), dim3(256), 0, st, a);
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
