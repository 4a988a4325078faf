// Selective scan: states whose decay and input the data choose, and its gradients.
//
// h_t = exp(d_t A) h_{t-1} + d_t x_t B_t: one exponential and four multiply-adds for each element of a state and step, against 8 bytes
// for each channel and step in 16 bits: with 16 elements a channel the exponentials (16 a clock and SM) bound it, not memory.
//
// Forwards a thread takes a channel, or two neighbouring ones, of one env through the steps, with 16 elements of the states in registers (channels
// with more of them belong to two or four lanes): nothing is shared but the rows of B and C, and a step's sum over the elements is the
// thread's own.  Backwards a thread has two elements of four channels, since there sums go over the channels as well as over the elements (four by
// four, or 16 of one channel, leave an SM 8 or 12 warps: 278 and 340 us where two by four take 264).  States, sums and arithmetic in 32 bits,
// packed arithmetic on two numbers at a time.
//
// Long sequences of few channels are cut into segments: a pass makes what each segment ends with, and each starts from the ends in front of it.
//
// Measured, channels of 16 elements in bf16: outputs of 16 steps of 256 envs of 2048 channels 68 us, 57 % of the rate of exponentials (134 MB in
// 21 us); of 8192 steps of 4096 channels 422 (in a profiler, one launch at a time: the pass over the segments 179 at 78 % of that rate, the
// outputs 262 at 64 %); gradients
// of the former 281, of 2048 steps of 2 envs of 2048 channels 396.
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
    long long ldx, lddt, ldb, ldc, ldz, ldy;  // from row to row, and from step to step:
    long long sx, st, sb, sc, sz, sy;
    int T, Be, channels, N, groups, per, softplus;  // per: channels of a group
    int tiles, group_tiles;                         // tiles of channels, in all and of a group
    int len, nseg;                                  // steps of a segment
    // Of every segment and env, [channels][NP] (N padded): the states it ends with (starting from zeros, but for the first one; in the last one's place
    // the state that comes in) and the gradients it hands to the steps in front (getting zeros; in the first one's place the gradient
    // of the state that is left); what its step sizes add up to for each channel, and whether a flag is set in it.
    float *seg, *back, *sum;
    int *cut;
    float *cum;     // BOTH: what the step sizes from the start of a segment add up to in front of every 16th step, [ceil(T / 16)][Be][channels]
    int *cum_cut;  // and whether a flag is set among them, [ceil(T / 16)][Be]
    float *mark;  // the states in front of every 16th step, [ceil(T / 16)][Be][channels][NP] (up to 16 steps: none)
    float *few;   // shares of the gradients of B and C, [group_tiles][T * Be][groups][2][NP]
    float *part;  // shares of the gradients of A, D and dt_bias, [parts][channels * (N + 2)]
    int parts;
};

// exp(d A), A times log2(e).  The hardware's exponential lies 0.4 units of 2^-24 too low on average for arguments between -0.5 and -0.01, which adds up over
// the hundreds of steps that a state remembers; with its argument moved by 2e-8 the mean is within 0.2 from -0.5 to 0 (one million arguments
// each), as near as expf's, at no cost.
constexpr float kShift = 2e-8f;
// A times log2(e); infinities give way to the largest numbers, so that they make 0 or infinity of any step size but 0, and 1 of that.
__device__ __forceinline__ float scaled(float A) {
    const float v = A * kLog2e;
    return isinf(v) ? copysignf(3e38f, v) : v;
}
__device__ __forceinline__ pair32 factors(pair32 d, pair32 A) { return exp2_pair(fma2(d, A, twice(kShift))); }
// h 2^(3 x) + add, the steps of a segment taken at once, a third of the way at a time: 2^(3 x) may leave the range where its product with h does not, and
// what is 0 stays 0 however much it would grow.  Beyond 2^360 the product leaves the range whatever h is.
__device__ __forceinline__ float carried(float x, float h, float add) {
    float y;
    asm("min.NaN.f32 %0, %1, 0f42F00000;" : "=f"(y) : "f"(x));  // 120
    const float f = exp2_fast(y);
    return fmaf(h * f * f, f, add);
}

// Sums of V values over LANES lanes, STRIDE apart: halves go to the lanes' halves as long as there are values, lane bit by lane bit from the
// highest; a lane is left with max(1, V / LANES) of them in v[0 ..], which ones spread_first says.
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

// Backwards NL lanes share four channels and hold two elements each of their states.
template <int NL>
struct Shape {
    static constexpr int NP = 2 * NL, GROUPS = 32 / NL, CT = 4 * GROUPS * (kThreads / 32);
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

// kSteps rows of a tile's channels on their way from memory: vectors of four elements, or single ones, dealt out to the threads.
template <typename T, int CT, bool VEC>
struct Rows {
    static constexpr int V = VEC ? 4 : 1, COLS = CT / V, PASSES = (kSteps * COLS + kThreads - 1) / kThreads;
    using Raw = std::conditional_t<VEC, std::conditional_t<sizeof(T) == 4, uint4, uint2>, T>;
    Raw raw[PASSES];
    static __device__ __forceinline__ int row(int i) { return (threadIdx.x + i * kThreads) / COLS; }
    static __device__ __forceinline__ int col(int i) { return (threadIdx.x + i * kThreads) % COLS * V; }
    // p: the tile's first channel in the env's row of step t
    __device__ __forceinline__ void fetch(const T *p, long long step, int rows, int cols) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (row(i) < min(rows, kSteps) && col(i) < cols) raw[i] = *reinterpret_cast<const Raw *>(p + row(i) * step + col(i));
    }
    // as pairs; of a single element the second is 0
    static constexpr int PAIRS = (V + 1) / 2;
    static __device__ __forceinline__ void get(const Raw &w, pair32 (&v)[PAIRS]) {
        if constexpr (VEC) {
            Vec<T> x;
            float f[Vec<T>::N];
            if constexpr (sizeof(T) == 4) x.raw = w;
            else x.raw = make_uint4(w.x, w.y, 0, 0);
            x.get(f);
            v[0] = pair_of(f[0], f[1]), v[1] = pair_of(f[2], f[3]);
        } else {
            v[0] = pair_of(to_f32(w), 0.f);
        }
    }
    static __device__ __forceinline__ void put(T *p, const pair32 (&v)[PAIRS]) {
        if constexpr (VEC) {
            const float2 a = parts(v[0]), b = parts(v[1]);
            float f[Vec<T>::N] = {a.x, a.y, b.x, b.y};
            Vec<T> x;
            x.set(f);
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(p) = x.raw;
            else *reinterpret_cast<uint2 *>(p) = make_uint2(x.raw.x, x.raw.y);
        } else {
            *p = from_f32<T>(parts(v[0]).x);
        }
    }
    // of 32-bit numbers in shared memory
    static __device__ __forceinline__ void put_shared(float *p, const pair32 (&v)[PAIRS]) {
        if constexpr (VEC) *reinterpret_cast<ulonglong2 *>(p) = make_ulonglong2(v[0], v[1]);
        else *p = parts(v[0]).x;
    }
    static __device__ __forceinline__ void get_shared(const float *p, pair32 (&v)[PAIRS]) {
        if constexpr (VEC) {
            const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p);
            v[0] = u.x, v[1] = u.y;
        } else {
            v[0] = pair_of(*p, 0.f);
        }
    }
    static __device__ __forceinline__ pair32 softplus(pair32 v) { return VEC ? softplus_pair(v) : pair_of(softplus_fast(parts(v).x), 0.f); }
    static __device__ __forceinline__ pair32 sigmoid(pair32 v) { return VEC ? sigmoid_pair(v) : pair_of(sigmoid_fast(parts(v).x), 0.f); }
};
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

// Elements n0 .. n0 + W - 1 of a state of N in memory, by vectors of four or two where these fit; zeros behind the last one.
template <int W>
__device__ __forceinline__ void load_row(const float *p, int N, int n0, float (&h)[W]) {
    constexpr int V = W % 4 == 0 ? 4 : 2;
    const bool whole = N % V == 0 && (reinterpret_cast<uintptr_t>(p) & (4 * V - 1)) == 0;
#pragma unroll
    for (int n = 0; n < W; n += V) {
        if (!whole) {
#pragma unroll
            for (int i = 0; i < V; ++i) h[n + i] = n0 + n + i < N ? p[n0 + n + i] : 0.f;
        } else if constexpr (V == 4) {
            const float4 f = n0 + n < N ? *reinterpret_cast<const float4 *>(p + n0 + n) : make_float4(0.f, 0.f, 0.f, 0.f);
            h[n] = f.x, h[n + 1] = f.y, h[n + 2] = f.z, h[n + 3] = f.w;
        } else {
            const float2 f = n0 + n < N ? *reinterpret_cast<const float2 *>(p + n0 + n) : make_float2(0.f, 0.f);
            h[n] = f.x, h[n + 1] = f.y;
        }
    }
}
template <int W>
__device__ __forceinline__ void store_row(float *p, int N, int n0, const float (&h)[W]) {
    constexpr int V = W % 4 == 0 ? 4 : 2;
    const bool whole = N % V == 0 && (reinterpret_cast<uintptr_t>(p) & (4 * V - 1)) == 0;
#pragma unroll
    for (int n = 0; n < W; n += V) {
        if (!whole) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n0 + n + i < N) p[n0 + n + i] = h[n + i];
        } else if (n0 + n < N) {
            if constexpr (V == 4) *reinterpret_cast<float4 *>(p + n0 + n) = make_float4(h[n], h[n + 1], h[n + 2], h[n + 3]);
            else *reinterpret_cast<float2 *>(p + n0 + n) = make_float2(h[n], h[n + 1]);
        }
    }
}
__device__ __forceinline__ void load_pairs(const float *p, pair32 (&v)[2]) {
    const ulonglong2 u = *reinterpret_cast<const ulonglong2 *>(p);
    v[0] = u.x, v[1] = u.y;
}

// Takes elements n0 .. of a channel's state, or gradient, through segment s: exp2(A sum of its step sizes) h + add, or add alone behind a flag.  from: what
// each segment adds; A: times log2(e).
template <int W>
__device__ __forceinline__ void through(const ScanArgs &a, int NP, int s, int e, int c, int n0, const float (&A)[W], const float *from, float (&h)[W]) {
    const long long at = (long long)s * a.Be + e;
    float add[W];
    load_row<W>(from + (at * a.channels + c) * NP, NP, n0, add);
    const bool cut = a.cut[at];
    const float d = a.sum[at * a.channels + c] * (1.f / 3);
#pragma unroll
    for (int n = 0; n < W; ++n) h[n] = cut ? add[n] : carried(d * A[n], h[n], add[n]);
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
#pragma unroll 4
    for (int s = a.nseg - 1; s > w.seg; --s) through<W>(a, NP, s, w.e, c, n0, A, a.back, g);
}

enum Mode {
    OUTPUT,  // y and the state that is left
    ENDS,    // what each segment ends with
    BOTH,    // that, the gradients it hands to the steps in front, and the states in front of every kSteps-th step (starting from zeros)
    MARKS    // the states in front of every kSteps-th step
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
__global__ void __launch_bounds__(kThreads, 4) scan_kernel(ScanArgs a) {
    grid_wait();
    constexpr int W = 16, P = W / 2, NP = W * NL, CT = kThreads / NL * CPT;
    constexpr bool WITH_C = MODE == OUTPUT || MODE == BOTH, WITH_DY = MODE == BOTH, WITH_Z = MODE == OUTPUT || MODE == BOTH;
    using Word = Cell<T, CPT>;
    __shared__ alignas(16) float sB[2][kSteps][NP], sC[2][WITH_C ? kSteps : 1][NP];
    const Work w = work_of<CT>(a, blockIdx.x % a.tiles, blockIdx.x / a.tiles);
    const int ln = threadIdx.x % NL, c = w.c0 + threadIdx.x / NL * CPT, n0 = ln * W;
    const bool on = c < w.c1;
    const long long &sx = a.sx, &st = a.st, &sb = a.sb, &sc = a.sc, &sz = a.sz, &sy = a.sy;
    const T *x = static_cast<const T *>(a.x) + w.e * a.ldx + c + w.t0 * sx, *dt = static_cast<const T *>(a.dt) + w.e * a.lddt + c + w.t0 * st;
    const T *B = static_cast<const T *>(a.B) + w.e * a.ldb + (long long)w.group * a.N + w.t0 * sb;
    const T *C = static_cast<const T *>(a.C) + w.e * a.ldc + (long long)w.group * a.N + w.t0 * sc;
    const T *z = WITH_Z && a.z ? static_cast<const T *>(a.z) + w.e * a.ldz + c + w.t0 * sz : nullptr;
    const T *dy = WITH_DY ? static_cast<const T *>(a.dy) + w.e * a.ldy + c + w.t0 * sy : nullptr;
    T *y = MODE == OUTPUT ? static_cast<T *>(a.y) + w.e * a.ldy + c + w.t0 * sy : nullptr;

    Word rx[4], rt[4], rz[WITH_Z ? 4 : 1], rg[WITH_DY ? 4 : 1];
    const auto fetch = [&](int k, bool there) {  // step k of the four at x, dt, z and dy
        if (!there) return;
        rx[k].load(x + k * sx);
        rt[k].load(dt + k * st);
        if (WITH_Z && z) rz[k].load(z + k * sz);
        if (WITH_DY) rg[k].load(dy + k * sy);
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) fetch(k, on && w.t0 + k < w.t1);
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
            for (int n = 0; n < W; ++n) Af[n] = scaled(Af[n]);
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
        if constexpr (MODE == MARKS || MODE == BOTH) {
            const long long at = (long long)(t / kSteps) * a.Be + w.e;
            float *to = a.mark + (at * a.channels + c) * NP + n0;
#pragma unroll
            for (int j = 0; j < CPT; ++j)
#pragma unroll
                for (int i = 0; i < P; i += 2)
                    if (on) *reinterpret_cast<ulonglong2 *>(to + j * NP + 2 * i) = make_ulonglong2(h[j][i], h[j][i + 1]);
            if constexpr (MODE == BOTH) {
                if (on && ln == 0) a.cum[at * a.channels + c] = parts(total).x;
                if (threadIdx.x == 0 && w.tile == 0) a.cum_cut[at] = cut;
            }
        }
#pragma unroll 1
        for (int s = 0; s < kSteps && s < rows; s += 4) {
            x += 4 * sx;
            dt += 4 * st;
            if (WITH_Z && z) z += 4 * sz;
            if (WITH_DY) dy += 4 * sy;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                pair32 xk = 0, dk = 0, zk = 0, gk = 0;  // steps behind the last one do nothing
                if (on && s + k < rows) {
                    xk = rx[k].get();
                    dk = add2(rt[k].get(), bias);
                    if (WITH_Z && z) zk = rz[k].get();
                    if (WITH_DY) gk = rg[k].get();
                }
                fetch(k, on && s + k + 4 < rows);  // the step that comes four steps later is on its way meanwhile
                if (a.softplus && on && s + k < rows) dk = Word::softplus(dk);
                if (WITH_Z && z) zk = Word::silu(zk);
                if (WITH_DY && z) gk = mul2(gk, zk);
                pair32 out[CPT];
                const float2 d = parts(dk), u = parts(mul2(dk, xk)), g = parts(gk);
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
                            const pair32 f = factors(twice(j == 0 ? d.x : d.y), A[j][i + m]);
                            h[j][i + m] = fma2(f, h[j][i + m], mul2(twice(j == 0 ? u.x : u.y), b[m]));
                            if constexpr (MODE == OUTPUT) out[j] = fma2(cc[m], h[j][i + m], out[j]);
                            if constexpr (WITH_DY) {
                                Pr[i + m] = mul2(Pr[i + m], f);
                                if (!cut) G[i + m] = fma2(mul2(Pr[i + m], twice(g.x)), cc[m], G[i + m]);
                            }
                        }
                }
                if constexpr (MODE == ENDS || MODE == BOTH) total = add2(total, dk);
                if constexpr (MODE == OUTPUT) {
                    const float2 o = parts(out[0]), q = parts(out[CPT - 1]);
                    float lo = o.x + o.y, hi = CPT == 2 ? q.x + q.y : 0.f;
#pragma unroll
                    for (int m = NL / 2; m > 0; m /= 2) {
                        lo += __shfl_xor_sync(0xffffffffu, lo, m);
                        if (CPT == 2) hi += __shfl_xor_sync(0xffffffffu, hi, m);
                    }
                    pair32 v = a.D ? fma2(D, xk, pair_of(lo, hi)) : pair_of(lo, hi);
                    if (z) v = mul2(v, zk);
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
            if (a.done && a.done[(long long)(w.t1 - 1) * a.Be + w.e]) {  // also where A is no number
#pragma unroll
                for (int n = 0; n < W; ++n) f[n] = 0.f;
            }
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

// The gradient that a segment hands to the steps in front, getting zeros, step by step from its last one: four elements of channel c.
template <typename T>
__device__ void handed(const ScanArgs &a, const Work &w, int c, int n0, const float (&A)[4], float (&g)[4]) {
    const int group = c / a.per;
#pragma unroll
    for (int n = 0; n < 4; ++n) g[n] = 0.f;
    for (int t = w.t1 - 1; t >= w.t0; --t) {
        if (a.done && a.done[(long long)t * a.Be + w.e]) {
#pragma unroll
            for (int n = 0; n < 4; ++n) g[n] = 0.f;
        }
        const T *C = static_cast<const T *>(a.C) + w.e * a.ldc + t * a.sc + (long long)group * a.N;
        float d = to_f32(static_cast<const T *>(a.dt)[w.e * a.lddt + t * a.st + c]) + (a.bias ? a.bias[c] : 0.f);
        float v = to_f32(static_cast<const T *>(a.dy)[w.e * a.ldy + t * a.sy + c]);
        if (a.softplus) d = softplus_fast(d);
        if (a.z) {
            const float z = to_f32(static_cast<const T *>(a.z)[w.e * a.ldz + t * a.sz + c]);
            v *= z * sigmoid_fast(z);
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (n0 + n < a.N) g[n] = fmaf(to_f32(C[n0 + n]), v, g[n]) * exp2_fast(fmaf(d, A[n], kShift));
    }
}

// The states in front of every kSteps-th step of the segments but the first, from those that started from zeros: what the segment starts from, taken
// through the steps in front of them, is added.  A thread has four elements of a channel in one segment.  It also looks at the gradient that the
// segment hands to the steps in front, a sum of products of factors forwards: where these have left the range, which leaves no finite sum, though the
// gradients of the steps need not have, it is made again.  (Where they fall below 2^-149 they count as 0.)
template <typename T>
__global__ void __launch_bounds__(256) scan_marks_kernel(ScanArgs a, int NP) {
    grid_wait();
    const int quads = NP / 4;
    const long long all = (long long)(a.nseg - 1) * a.Be * a.channels * quads, id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= all) return;
    const long long chan = id / quads, item = chan / a.channels;
    const int n0 = (int)(id - chan * quads) * 4, c = (int)(chan - item * a.channels);
    Work w = {};
    w.seg = (int)(item / a.Be) + 1;
    w.e = (int)(item % a.Be);
    w.t0 = w.seg * a.len;
    w.t1 = min(a.T, w.t0 + a.len);
    float A[4], h[4], f[4], g[4];
    load_row<4>(a.A + (long long)c * a.N, a.N, n0, A);
#pragma unroll
    for (int n = 0; n < 4; ++n) A[n] = scaled(A[n]);
    float *back = a.back + (((long long)w.seg * a.Be + w.e) * a.channels + c) * NP;
    load_row<4>(back, NP, n0, g);
    start_of<4>(a, NP, w, c, n0, A, h);
    for (int t = w.t0; t < w.t1; t += kSteps) {
        const long long at = (long long)(t / kSteps) * a.Be + w.e;
        if (a.cum_cut[at]) break;
        const float d = a.cum[at * a.channels + c] * (1.f / 3);
        float *mark = a.mark + (at * a.channels + c) * NP;
        load_row<4>(mark, NP, n0, f);
#pragma unroll
        for (int n = 0; n < 4; ++n) f[n] = carried(d * A[n], h[n], f[n]);
        store_row<4>(mark, NP, n0, f);
    }
    if (isfinite(g[0]) && isfinite(g[1]) && isfinite(g[2]) && isfinite(g[3])) return;
    handed<T>(a, w, c, n0, A, h);
#pragma unroll
    for (int n = 0; n < 4; ++n) g[n] = isfinite(g[n]) ? g[n] : h[n];
    store_row<4>(back, NP, n0, g);
}

// Gradients.  Per step, with g = dL/dh_t and dv = dL/dy silu(z):
//   g_t = C_t dv_t + (nothing where done[t] is set, else) exp(d_{t+1} A) g_{t+1},   q = g_t exp(d_t A) h'_{t-1}
//   dC = sum_c dv h,  dB = sum_c g d x,  dx = D dv + d sum_n g B,  dd = x sum_n g B + sum_n q A,  dA += q d
// Sixteen steps at a time, from the last ones to the first: forwards once from the states in front of them, which leaves those in front of every
// fourth step; then four steps at a time, backwards: forwards through them, which leaves exp(d A) h' of the four in registers (and y and
// the sums of dC on the way), and backwards over these, where the factors are made a second time: kept, they would take the registers of
// half the warps.  A block goes through as many envs, or segments, as fall to it, copies the rows of the next sixteen steps ahead while it works,
// and keeps its shares of the parameters' gradients.  16 steps of 256 envs of 2048 x 16 bf16: 277 us in a profiler, 57 % of the issue
// slots (620 instructions for 32 channels of a step, a third of them integer arithmetic and selections around the sums over lanes; 128 registers,
// as many as four blocks an SM leave, and 52 bytes a thread beside them in local memory).

// Two elements of the states of four channels, [e][channel][N] in memory; zeros where there are none.
__device__ __forceinline__ void load_block(const float *from, const ScanArgs &a, int e, int c, int c1, int n0, float (&h)[4][2]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j][0] = h[j][1] = 0.f;
        if (from && c + j < c1) load_row<2>(from + ((long long)e * a.channels + c + j) * a.N, a.N, n0, h[j]);
    }
}
__device__ __forceinline__ void store_block(float *to, const ScanArgs &a, int e, int c, int c1, int n0, const float (&h)[4][2]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (c + j < c1) store_row<2>(to + ((long long)e * a.channels + c + j) * a.N, a.N, n0, h[j]);
}
// As pairs of neighbouring channels.
__device__ __forceinline__ void pack(const float (&h)[4][2], pair32 (&p)[2][2]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) p[n][0] = pair_of(h[0][n], h[1][n]), p[n][1] = pair_of(h[2][n], h[3][n]);
}
__device__ __forceinline__ void unpack(const pair32 (&p)[2][2], float (&h)[4][2]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const float2 u = parts(p[n][0]), v = parts(p[n][1]);
        h[0][n] = u.x, h[1][n] = u.y, h[2][n] = v.x, h[3][n] = v.y;
    }
}

template <typename T, int NL, bool VEC>
struct GradShared {
    static constexpr int CT = Shape<NL>::CT, NP = Shape<NL>::NP;
    using R = Rows<T, CT, VEC>;
    float sd[kSteps][CT], su[kSteps][CT], sg[kSteps][CT], sy[kSteps][CT], sD[CT], sbias[CT];
    float2 sB[kSteps][NP], sC[kSteps][NP];  // every element twice, as packed arithmetic on two channels takes it
    float few[kThreads / 32][kSteps][2 * NP];
    // a thread's own: the states in front of the tile, and of its steps 4 and 8 (from 12 on they start where the way forwards ends); its sums of
    // the gradients of D and dt_bias; its elements of the next tile's rows of x, dt, dy, z
    float2 mark[4][kThreads];
    float4 inner[2][2][kThreads];
    float kept[2][kThreads * R::V];
    typename R::Raw next[4][R::PASSES][kThreads];
};

// BYTES of them, or zeros.
template <int BYTES>
__device__ __forceinline__ void copy_async(void *to, const void *from, bool there) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 2) {
        if (there) *static_cast<uint16_t *>(to) = *static_cast<const uint16_t *>(from);
    } else {
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(at), "l"(from), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
    }
}

template <typename T, int NL, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) scan_bwd_kernel(ScanArgs a) {
    grid_wait();
    constexpr int NPT = 2;
    using S = Shape<NL>;
    constexpr int CT = S::CT, NP = S::NP, GROUPS = S::GROUPS, FEW = kSteps * NP / kThreads;
    using R = Rows<T, CT, VEC>;
    constexpr int BYTES = sizeof(typename R::Raw);
    extern __shared__ __align__(16) char smem[];
    GradShared<T, NL, VEC> &s = *reinterpret_cast<GradShared<T, NL, VEC> *>(smem);
    const int tile = blockIdx.x % a.tiles, slice = blockIdx.x / a.tiles;
    const int lane = threadIdx.x % 32, ln = lane % NL, warp = threadIdx.x / 32, n0 = ln * NPT, local = (warp * GROUPS + lane / NL) * 4;
    Work w = work_of<CT>(a, tile, slice);
    const int c = w.c0 + local, cols = w.c1 - w.c0;
    const long long &sx = a.sx, &st = a.st, &sb = a.sb, &sc = a.sc, &sz = a.sz, &sy = a.sy;
    pair32 A[NPT][2], g[NPT][2], dA[NPT][2];
    {
        float f[4][NPT];
        load_block(a.A, a, 0, c, w.c1, n0, f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int n = 0; n < NPT; ++n) f[j][n] = scaled(f[j][n]);
        pack(f, A);
#pragma unroll
        for (int n = 0; n < NPT; ++n) dA[n][0] = dA[n][1] = 0;
    }
    stage_channels(s.sD, a.D, w);
    stage_channels(s.sbias, a.bias, w);
#pragma unroll
    for (int v = 0; v < R::V; ++v) s.kept[0][threadIdx.x * R::V + v] = s.kept[1][threadIdx.x * R::V + v] = 0.f;

    // of the tile that comes next
    T fb[FEW], fc[FEW];
    const auto fetch = [&](const Work &w, int t) {
        const int rows = min(w.t1 - t, kSteps);
        const T *x = static_cast<const T *>(a.x) + w.e * a.ldx + w.c0 + t * sx, *dt = static_cast<const T *>(a.dt) + w.e * a.lddt + w.c0 + t * st;
        const T *dy = static_cast<const T *>(a.dy) + w.e * a.ldy + w.c0 + t * sy, *z = a.z ? static_cast<const T *>(a.z) + w.e * a.ldz + w.c0 + t * sz : nullptr;
#pragma unroll
        for (int i = 0; i < R::PASSES; ++i) {
            const int r = R::row(i), l = R::col(i);
            if (r >= rows || l >= cols) continue;
            copy_async<BYTES>(&s.next[0][i][threadIdx.x], x + r * sx + l, true);
            copy_async<BYTES>(&s.next[1][i][threadIdx.x], dt + r * st + l, true);
            copy_async<BYTES>(&s.next[2][i][threadIdx.x], dy + r * sy + l, true);
            if (z) copy_async<BYTES>(&s.next[3][i][threadIdx.x], z + r * sz + l, true);
        }
        const T *B = static_cast<const T *>(a.B) + w.e * a.ldb + (long long)w.group * a.N + t * sb;
        const T *C = static_cast<const T *>(a.C) + w.e * a.ldc + (long long)w.group * a.N + t * sc;
#pragma unroll
        for (int i = 0; i < FEW; ++i) {
            const int r = threadIdx.x / NP + i * (kThreads / NP), n = threadIdx.x % NP;
            const bool ok = r < rows && n < a.N;
            fb[i] = ok ? B[r * sb + n] : from_f32<T>(0.f);
            fc[i] = ok ? C[r * sc + n] : from_f32<T>(0.f);
        }
    };
    const auto fetch_mark = [&](const Work &w, int t) {
        // up to kSteps steps start from the state that comes in, whose rows need not be aligned
        const float *mark = a.mark + (((long long)(t / kSteps) * a.Be + w.e) * a.channels + c) * NP + n0;
        if (a.T > kSteps) {
#pragma unroll
            for (int j = 0; j < 4; ++j) copy_async<8>(&s.mark[j][threadIdx.x], c + j < w.c1 ? mark + j * NP : a.mark, c + j < w.c1);
        } else {
            float f[4][NPT];
            load_block(a.state_in, a, w.e, c, w.c1, n0, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) s.mark[j][threadIdx.x] = make_float2(f[j][0], f[j][1]);
        }
    };
    const auto last_tile = [&](const Work &w) { return w.t0 + (w.t1 - 1 - w.t0) / kSteps * kSteps; };
    fetch(w, last_tile(w));
    fetch_mark(w, last_tile(w));

    const long long items = (long long)a.Be * a.nseg;
    for (long long item = slice; item < items; item += a.parts) {
        w = work_of<CT>(a, tile, item);
        {
            float f[4][NPT], Af[4][NPT];
            if (a.nseg == 1) {
                load_block(a.dstate_out, a, w.e, c, w.c1, n0, f);
            } else {
                unpack(A, Af);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    f[j][0] = f[j][1] = 0.f;
                    if (c + j < w.c1) end_of<2>(a, NP, w, c + j, n0, Af[j], f[j]);
                }
            }
            pack(f, g);
        }
        for (int t = last_tile(w); t >= w.t0; t -= kSteps) {
            // A last tile's rows are moved behind up to three rows of zeros, so that they end with a whole group of four: steps of size 0 in front of the
            // first one hand its state and its gradient through, and no gradient passes any behind the last one, which may drop it.
            const int rows = min(w.t1 - t, kSteps), pad = -rows & 3;
            const auto place = [pad](int r) { return (r + pad) & (kSteps - 1); };
            const uint32_t flag = flags_of(a, w.e, t, rows) << pad;
            __syncthreads();  // the tile behind is done with
            asm volatile("cp.async.wait_all;" ::: "memory");  // a thread reads what it copied itself
#pragma unroll
            for (int i = 0; i < FEW; ++i) {
                const int r = threadIdx.x / NP + i * (kThreads / NP), n = threadIdx.x % NP;
                const float b = to_f32(fb[i]), f = to_f32(fc[i]);
                s.sB[place(r)][n] = make_float2(b, b);
                s.sC[place(r)][n] = make_float2(f, f);
            }
#pragma unroll
            for (int i = 0; i < R::PASSES; ++i) {
                const int r = R::row(i), l = R::col(i);
                pair32 d[R::PAIRS] = {}, u[R::PAIRS] = {}, v[R::PAIRS] = {};
                if (r < rows && l < cols) {
                    pair32 b[R::PAIRS];
                    R::get(s.next[0][i][threadIdx.x], u);
                    R::get(s.next[1][i][threadIdx.x], d);
                    R::get(s.next[2][i][threadIdx.x], v);
                    R::get_shared(&s.sbias[l], b);
#pragma unroll
                    for (int k = 0; k < R::PAIRS; ++k) {
                        d[k] = add2(d[k], b[k]);
                        if (a.softplus) d[k] = R::softplus(d[k]);
                        u[k] = mul2(u[k], d[k]);
                    }
                    if (a.z) {
                        pair32 f[R::PAIRS];
                        R::get(s.next[3][i][threadIdx.x], f);
#pragma unroll
                        for (int k = 0; k < R::PAIRS; ++k) v[k] = mul2(v[k], mul2(f[k], R::sigmoid(f[k])));
                    }
                }
                if (r >= kSteps) break;
                R::put_shared(&s.sd[place(r)][l], d);
                R::put_shared(&s.su[place(r)][l], u);
                R::put_shared(&s.sg[place(r)][l], v);
            }
            {
                // on its way while this tile is worked on
                const bool more = t > w.t0;
                if (more || item + a.parts < items) {
                    const Work v = more ? w : work_of<CT>(a, tile, item + a.parts);
                    fetch(v, more ? t - kSteps : last_tile(v));
                }
            }
            __syncthreads();
            const int top = (rows - 1) / 4;
            pair32 h[NPT][2];
            const auto load_start = [&](int m) {  // the states in front of steps 4 m ..
                if (m == 0) {
                    float f[4][NPT];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 v = s.mark[j][threadIdx.x];
                        f[j][0] = v.x, f[j][1] = v.y;
                    }
                    pack(f, h);
                } else {
#pragma unroll
                    for (int n = 0; n < NPT; ++n) {
                        const float4 f = s.inner[m - 1][n][threadIdx.x];
                        h[n][0] = pair_of(f.x, f.y), h[n][1] = pair_of(f.z, f.w);
                    }
                }
            };
            load_start(0);
            // forwards to the states in front of every fourth step
#pragma unroll 1
            for (int m = 0; m < top; ++m) {
                if (m > 0) s.inner[m - 1][0][threadIdx.x] = make_float4(parts(h[0][0]).x, parts(h[0][0]).y, parts(h[0][1]).x, parts(h[0][1]).y);
                if (m > 0) s.inner[m - 1][1][threadIdx.x] = make_float4(parts(h[1][0]).x, parts(h[1][0]).y, parts(h[1][1]).x, parts(h[1][1]).y);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = 4 * m + k;
                    pair32 d[2], u[2], b[2];
                    load_pairs(&s.sd[r][local], d);
                    load_pairs(&s.su[r][local], u);
                    load_pairs(&s.sB[r][n0].x, b);
#pragma unroll
                    for (int n = 0; n < NPT; ++n)
#pragma unroll
                        for (int p = 0; p < 2; ++p) h[n][p] = fma2(factors(d[p], A[n][p]), h[n][p], mul2(u[p], b[n]));
                    if (flag >> r & 1) {
#pragma unroll
                        for (int n = 0; n < NPT; ++n) h[n][0] = h[n][1] = 0;
                    }
                }
            }
#pragma unroll 1
            for (int m = top; m >= 0; --m) {
                const int r0 = 4 * m;
                if (m < top) load_start(m);
                pair32 q[4][NPT][2];  // of each step exp(d A) times the state in front
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    float ys[8], cs[4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r = r0 + k + i;
                        pair32 d[2], u[2], v[2], acc[2] = {0, 0}, b[2], cc[2];
                        load_pairs(&s.sd[r][local], d);
                        load_pairs(&s.su[r][local], u);
                        load_pairs(&s.sg[r][local], v);
                        load_pairs(&s.sB[r][n0].x, b);
                        load_pairs(&s.sC[r][n0].x, cc);
                        if (k + i > 0 && flag >> (r - 1) & 1) {
#pragma unroll
                            for (int n = 0; n < NPT; ++n) h[n][0] = h[n][1] = 0;
                        }
#pragma unroll
                        for (int n = 0; n < NPT; ++n) {
                            pair32 sum = 0;
#pragma unroll
                            for (int p = 0; p < 2; ++p) {
                                const pair32 qq = mul2(factors(d[p], A[n][p]), h[n][p]);
                                q[k + i][n][p] = qq;
                                h[n][p] = fma2(u[p], b[n], qq);
                                acc[p] = fma2(cc[n], h[n][p], acc[p]);
                                sum = fma2(v[p], h[n][p], sum);
                            }
                            const float2 e = parts(sum);
                            cs[2 * i + n] = e.x + e.y;
                        }
                        const float2 e = parts(acc[0]), o = parts(acc[1]);
                        ys[4 * i] = e.x, ys[4 * i + 1] = e.y, ys[4 * i + 2] = o.x, ys[4 * i + 3] = o.y;
                    }
                    if (a.z) {
                        spread_sum<8, NL, 1>(ys, lane);
                        const int at = spread_first<8, NL>(ln);
                        s.sy[r0 + k + at / 4][local + at % 4] = ys[0];
                    }
                    spread_sum<4, GROUPS, NL>(cs, lane);
                    const int at = spread_first<4, GROUPS>(lane / NL);
#pragma unroll
                    for (int i = 0; i < 4 / GROUPS; ++i) s.few[warp][r0 + k + (at + i) / 2][NP + n0 + (at + i) % 2] = cs[i];
                }
#pragma unroll
                for (int k = 2; k >= 0; k -= 2) {
                    float bs[4];
#pragma unroll
                    for (int i = 1; i >= 0; --i) {
                        const int r = r0 + k + i;
                        pair32 d[2], u[2], v[2], s1[2] = {0, 0}, s2[2] = {0, 0}, b[2], cc[2];
                        load_pairs(&s.sd[r][local], d);
                        load_pairs(&s.su[r][local], u);
                        load_pairs(&s.sg[r][local], v);
                        load_pairs(&s.sB[r][n0].x, b);
                        load_pairs(&s.sC[r][n0].x, cc);
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
                                g[n][p] = mul2(g[n][p], factors(d[p], A[n][p]));
                            }
                            const float2 e = parts(sum);
                            bs[2 * i + n] = e.x + e.y;
                        }
                        float both[8];
                        const float2 e = parts(s1[0]), o = parts(s1[1]), e2 = parts(s2[0]), o2 = parts(s2[1]);
                        both[0] = e.x, both[1] = e.y, both[2] = o.x, both[3] = o.y;
                        both[4] = e2.x, both[5] = e2.y, both[6] = o2.x, both[7] = o2.y;
                        spread_sum<8, NL, 1>(both, lane);
                        const int at = spread_first<8, NL>(ln);
                        __syncwarp();  // every lane of the channels has read this step's row: the sums take its place
                        *((at < 4 ? &s.su[r][local] : &s.sg[r][local - 4]) + at) = both[0];
                    }
                    spread_sum<4, GROUPS, NL>(bs, lane);
                    const int at = spread_first<4, GROUPS>(lane / NL);
#pragma unroll
                    for (int i = 0; i < 4 / GROUPS; ++i) s.few[warp][r0 + k + (at + i) / 2][n0 + (at + i) % 2] = bs[i];
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < kSteps * 2 * NP; i += kThreads) {
                const int r = i / (2 * NP), n = i % (2 * NP);
                if (r >= rows) break;
                float sum = 0.f;
#pragma unroll
                for (int k = 0; k < kThreads / 32; ++k) sum += s.few[k][place(r)][n];
                const long long row = (long long)(t + r) * a.Be + w.e;
                a.few[(((long long)(tile - w.group * a.group_tiles) * a.T * a.Be + row) * a.groups + w.group) * (2 * NP) + n] = sum;
            }
            if (const bool more = t > w.t0; more || item + a.parts < items) {
                const Work v = more ? w : work_of<CT>(a, tile, item + a.parts);
                fetch_mark(v, more ? t - kSteps : last_tile(v));
            }
            {
                const long long ax = w.e * a.ldx + w.c0 + t * sx, at = w.e * a.lddt + w.c0 + t * st, az = w.e * a.ldz + w.c0 + t * sz, ay = w.e * a.ldy + w.c0 + t * sy;
                R rx, rt, rg, rz;
                rx.fetch(static_cast<const T *>(a.x) + ax, sx, rows, cols);
                rt.fetch(static_cast<const T *>(a.dt) + at, st, rows, cols);
                rg.fetch(static_cast<const T *>(a.dy) + ay, sy, rows, cols);
                if (a.z) rz.fetch(static_cast<const T *>(a.z) + az, sz, rows, cols);
                T *dx = static_cast<T *>(a.dx) + ax, *ddt = static_cast<T *>(a.ddt) + at, *dz = a.z ? static_cast<T *>(a.dz) + az : nullptr;
                pair32 D[R::PAIRS], bias[R::PAIRS], sumD[R::PAIRS], sumb[R::PAIRS];
                float *keptD = &s.kept[0][threadIdx.x * R::V], *keptb = &s.kept[1][threadIdx.x * R::V];
                R::get_shared(&s.sD[R::col(0)], D);  // every pass has the same columns
                R::get_shared(&s.sbias[R::col(0)], bias);
                R::get_shared(keptD, sumD);
                R::get_shared(keptb, sumb);
#pragma unroll
                for (int i = 0; i < R::PASSES; ++i) {
                    const int r = R::row(i), l = R::col(i);
                    if (r >= rows || l >= cols) continue;
                    pair32 d[R::PAIRS], s1[R::PAIRS], s2[R::PAIRS], xv[R::PAIRS], tv[R::PAIRS], gv[R::PAIRS], o[R::PAIRS];
                    R::get_shared(&s.sd[place(r)][l], d);
                    R::get_shared(&s.su[place(r)][l], s1);
                    R::get_shared(&s.sg[place(r)][l], s2);
                    R::get(rx.raw[i], xv);
                    R::get(rt.raw[i], tv);
                    R::get(rg.raw[i], gv);
                    if (a.z) {
                        pair32 zv[R::PAIRS], yv[R::PAIRS];
                        R::get(rz.raw[i], zv);
                        R::get_shared(&s.sy[place(r)][l], yv);
#pragma unroll
                        for (int k = 0; k < R::PAIRS; ++k) {
                            const pair32 p = R::sigmoid(zv[k]), all = a.D ? fma2(D[k], xv[k], yv[k]) : yv[k], one = twice(1.f);
                            o[k] = mul2(gv[k], mul2(all, mul2(p, fma2(zv[k], fma2(p, twice(-1.f), one), one))));
                            gv[k] = mul2(gv[k], mul2(zv[k], p));
                        }
                        R::put(dz + r * sz + l, o);
                    }
#pragma unroll
                    for (int k = 0; k < R::PAIRS; ++k) {
                        o[k] = mul2(d[k], s1[k]);
                        if (a.D) o[k] = fma2(D[k], gv[k], o[k]);
                        sumD[k] = fma2(gv[k], xv[k], sumD[k]);
                    }
                    R::put(dx + r * sx + l, o);
#pragma unroll
                    for (int k = 0; k < R::PAIRS; ++k) {
                        o[k] = fma2(xv[k], s1[k], mul2(twice(kLn2), s2[k]));
                        if (a.softplus) o[k] = mul2(o[k], R::sigmoid(add2(tv[k], bias[k])));
                        sumb[k] = add2(sumb[k], o[k]);
                    }
                    R::put(ddt + r * st + l, o);
                }
                R::put_shared(keptD, sumD);
                R::put_shared(keptb, sumb);
            }
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
        unpack(dA, f);
        store_block(part, a, 0, c, w.c1, n0, f);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * CT; i += kThreads) {
        const int k = i / CT, l = i % CT;
        if (l >= cols) continue;
        float sum = 0.f;
        for (int r = 0; r < kThreads / R::COLS; ++r) sum += s.kept[k][(r * R::COLS + l / R::V) * R::V + l % R::V];
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

// One step, the state in place: NL lanes share four channels of a group, four elements of each, whose step sizes and outputs they share out among
// them.  Bound by memory, since the states go through once: a thread copies its own of the next envs ahead into shared memory, and reads
// the next env's rows while it works on this one's.  512 envs of 4096 x 16: 55 us, 5.2 TB/s (one channel a thread, 4 KB side by side: 82).
constexpr int kAhead = 3;  // envs in the ring

template <typename T, int NL>
__global__ void __launch_bounds__(256, 3) scan_step_kernel(ScanArgs a, int envs) {
    grid_wait();
    constexpr int CH = 256 / NL, LEFT = NL >= 4 ? 1 : 4 / NL, EACH = NL >= 4 ? NL / 4 : 1;  // channels side by side; of a lane's own; lanes of one
    extern __shared__ float4 ring[][4][256];
    const int cols = (a.per + 4 * CH - 1) / (4 * CH), col = blockIdx.x % (cols * a.groups), group = col / cols;
    const int c = group * a.per + col % cols * 4 * CH + threadIdx.x / NL, end = (group + 1) * a.per, ln = threadIdx.x % NL, n0 = ln * 4;
    const int e0 = blockIdx.x / (cols * a.groups) * envs, e1 = min(a.Be, e0 + envs), first = ln / EACH * LEFT;
    const bool whole = a.N % 4 == 0, ahead = whole && n0 < a.N;
    const bool few = whole && ((a.ldb | a.ldc) & 3) == 0 && ((reinterpret_cast<uintptr_t>(a.B) | reinterpret_cast<uintptr_t>(a.C)) & (4 * sizeof(T) - 1)) == 0;
    const long long next = (long long)a.channels * a.N;
    const int apart = CH * a.N;  // from one of the four channels to the next
    // of the envs that are copied ahead, read, and written next
    float *state = a.state_out + ((long long)e0 * a.channels + c) * a.N + n0;
    const float *to_copy = state;
    const T *B = static_cast<const T *>(a.B) + e0 * a.ldb + (long long)group * a.N + n0, *C = static_cast<const T *>(a.C) + e0 * a.ldc + (long long)group * a.N + n0;
    const int own = c + first * CH;  // the first of the channels that are this lane's
    const T *xp = static_cast<const T *>(a.x) + e0 * a.ldx + own, *tp = static_cast<const T *>(a.dt) + e0 * a.lddt + own;
    const T *zp = static_cast<const T *>(a.z) + e0 * a.ldz + own;
    T *yp = static_cast<T *>(a.y) + e0 * a.ldy + own;
    const uint8_t *done = a.done + e0;
    int copied = e0, slot_to = 0;
    const auto fetch = [&] {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (ahead && copied < e1 && c + j * CH < end) {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(&ring[slot_to][j][threadIdx.x]);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(to_copy + j * apart) : "memory");
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ++copied;
        to_copy += next;
        slot_to = slot_to == kAhead - 1 ? 0 : slot_to + 1;
    };
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i) fetch();
    using Four = std::conditional_t<sizeof(T) == 4, uint4, uint2>;
    const auto load_four = [&](const T *p) {
        Four w = {};
        if (few) {
            if (n0 < a.N) w = *reinterpret_cast<const Four *>(p);
        } else {
            T *v = reinterpret_cast<T *>(&w);
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = n0 + n < a.N ? p[n] : from_f32<T>(0.f);
        }
        return w;
    };
    const auto floats = [](const Four &w, float (&v)[4]) {
        Vec<T> r;
        float f[Vec<T>::N];
        if constexpr (sizeof(T) == 4) r.raw = w;
        else r.raw = make_uint4(w.x, w.y, 0, 0);
        r.get(f);
#pragma unroll
        for (int n = 0; n < 4; ++n) v[n] = f[n];
    };
    Four rb, rc;
    T rx[LEFT], rt[LEFT], rz[LEFT];
    bool empty = false;
    const auto read = [&](int e) {
        if (e >= e1) return;
        empty = a.done && *done;
        rb = load_four(B);
        rc = load_four(C);
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            if (own + i * CH >= end) break;
            rx[i] = xp[i * CH];
            rt[i] = tp[i * CH];
            if (a.z) rz[i] = zp[i * CH];
        }
        B += a.ldb, C += a.ldc, xp += a.ldx, tp += a.lddt, zp += a.ldz, ++done;
    };
    read(e0);
    float A[4][4], D[LEFT], bias[LEFT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int n = 0; n < 4; ++n) A[j][n] = 0.f;
        if (c + j * CH < end) load_row<4>(a.A + (long long)(c + j * CH) * a.N, a.N, n0, A[j]);
#pragma unroll
        for (int n = 0; n < 4; ++n) A[j][n] = scaled(A[j][n]);
    }
#pragma unroll
    for (int i = 0; i < LEFT; ++i) {
        D[i] = a.D && own + i * CH < end ? a.D[own + i * CH] : 0.f;
        bias[i] = a.bias && own + i * CH < end ? a.bias[own + i * CH] : 0.f;
    }
    int slot = 0;
    for (int e = e0; e < e1; ++e, slot = slot == kAhead - 1 ? 0 : slot + 1, state += next, yp += a.ldy) {
        fetch();
        float b[4], cc[4], x[LEFT] = {}, z[LEFT] = {}, d[LEFT] = {}, y[4];
        const bool start = empty;
        floats(rb, b);
        floats(rc, cc);
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            if (own + i * CH >= end) break;
            x[i] = to_f32(rx[i]);
            d[i] = to_f32(rt[i]) + bias[i];
            if (a.z) z[i] = to_f32(rz[i]);
        }
        read(e + 1);
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < LEFT; ++i) d[i] = softplus_fast(d[i]);
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float dj = __shfl_sync(0xffffffffu, d[j % LEFT], j / LEFT * EACH, NL), uj = __shfl_sync(0xffffffffu, d[j % LEFT] * x[j % LEFT], j / LEFT * EACH, NL);
            float h[4] = {};
            y[j] = 0.f;
            if (c + j * CH >= end) continue;
            if (!start) {
                if (ahead) {
                    const float4 f = ring[slot][j][threadIdx.x];
                    h[0] = f.x, h[1] = f.y, h[2] = f.z, h[3] = f.w;
                } else if (!whole) {
                    load_row<4>(state - n0 + j * apart, a.N, n0, h);
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                h[n] = fmaf(exp2_fast(fmaf(dj, A[j][n], kShift)), h[n], uj * b[n]);
                y[j] = fmaf(cc[n], h[n], y[j]);
            }
            if (ahead) *reinterpret_cast<float4 *>(state + j * apart) = make_float4(h[0], h[1], h[2], h[3]);
            else if (!whole) store_row<4>(state - n0 + j * apart, a.N, n0, h);
        }
        spread_sum<4, NL, 1>(y, ln);
#pragma unroll
        for (int i = 0; i < LEFT; ++i) {
            if (own + i * CH >= end || ln % EACH != 0) break;
            float v = a.D ? fmaf(D[i], x[i], y[i]) : y[i];
            if (a.z) v *= z[i] * sigmoid_fast(z[i]);
            yp[i * CH] = from_f32<T>(v);
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
    size_t seg, sums, mark, cum, few, part;  // floats of each area of the workspace
};
Plan plan_of(const ppo_selective_scan_desc *d, bool bwd) {
    Plan p = {};
    p.NL = d->N <= 16 ? 1 : d->N <= 32 ? 2 : 4;
    p.NP = 16 * p.NL;
    const auto up = [](size_t n) { return (n + 7) & ~(size_t)7; };  // whole 32 bytes
    const int per = d->channels / d->groups;
    p.group_tiles = ppo_cdiv(per, 64 / p.NL);
    p.tiles = p.group_tiles * d->groups;
    // segments: forwards as many as fill four blocks an SM; backwards, where three passes go over them, as many as deal two to each slice of blocks;
    // none shorter than 32 steps (gradients of 119 steps of 37 envs of 202 channels: 110 us with 64, 94 with 32, 95 with 16), no more than 64, since
    // each starts by going through those in front of it (8192 steps of 512 channels: 165 us with 32 of them, 115 with 64, 113 with 96, 483 with 256)
    const int room = (d->dtype == PPO_F32 ? 3 : 4) * 148, slices = p.tiles < room ? room / p.tiles : 1;  // one round of scan_bwd_kernel's blocks
    const long long blocks = (long long)d->Be * d->groups * ppo_cdiv(per, 256 / p.NL);
    long long n = bwd ? (d->Be < slices ? 2ll * slices / d->Be : 1) : (blocks < 4 * 148 ? 4 * 148 / blocks : 1);
    const int most = ppo_cdiv(d->T, 32);
    if (n > most) n = most;
    if (n > 64) n = 64;
    p.len = ppo_cdiv(ppo_cdiv(d->T, n), kSteps) * kSteps;
    p.nseg = ppo_cdiv(d->T, p.len);
    const size_t held = (size_t)d->Be * d->channels * p.NP;
    if (p.nseg > 1) {
        p.seg = p.nseg * held;
        p.sums = up((size_t)p.nseg * d->Be * (d->channels + 1));
    }
    if (bwd) {
        p.mark = d->T > kSteps ? ppo_cdiv(d->T, kSteps) * held : 0;
        p.cum = p.nseg > 1 ? up((size_t)ppo_cdiv(d->T, kSteps) * d->Be * (d->channels + 1)) : 0;
        p.few = (size_t)d->T * d->Be * p.tiles * 2 * p.NP;
        const long long items = (long long)d->Be * p.nseg;
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
    a.sx = d->Be * d->ldx;
    a.st = d->Be * d->lddt;
    a.sb = d->Be * d->ldb;
    a.sc = d->Be * d->ldc;
    a.sz = d->Be * d->ldz;
    a.sy = d->Be * d->ldy;
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
// A pass over the first `segs` segments, CPT channels a thread.
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
    // one channel a thread where two would leave SMs with less than two blocks
    two = two && (long long)a.Be * a.groups * ppo_cdiv(a.per, kThreads / NL * 2) * segs >= 2 * 148;
    return two ? pass_of<T, NL, 2, MODE>(a, segs, st) : pass_of<T, NL, 1, MODE>(a, segs, st);
}

}  // namespace

extern "C" size_t ppo_selective_scan_workspace_bytes(const ppo_selective_scan_desc *d, int backward) {
    if (check(d) != PPO_OK) return 0;
    const Plan p = plan_of(d, backward != 0);
    return ((backward ? 2 : 1) * p.seg + p.sums + p.mark + p.cum + p.few + p.part) * sizeof(float);
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
    a.cum = a.mark + p.mark;
    a.cum_cut = reinterpret_cast<int *>(a.cum + (size_t)ppo_cdiv(d->T, kSteps) * d->Be * d->channels);
    a.few = a.cum + p.cum;
    const bool params = dA || dD || ddt_bias;
    a.part = params ? a.few + p.few : nullptr;
    a.sum = a.few + p.few + p.part;
    a.cut = reinterpret_cast<int *>(a.sum + (size_t)p.nseg * d->Be * d->channels);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool two = vectors(d, 2, {x, dt}), vec = vectors(d, 4, {x, dt, z, dy, dx, ddt, dz});
    PPO_TRY(with_lanes(d, p, [&](auto t, auto nl) -> int {
        using T = decltype(t);
        constexpr int NL = decltype(nl)::value;
        if (p.nseg > 1) {
            PPO_TRY((pass_of<T, NL, 1, BOTH>(a, p.nseg, st)));
            const long long quads = (long long)(p.nseg - 1) * d->Be * d->channels * (p.NP / 4);
            PPO_TRY(ppo_launch(scan_marks_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a, p.NP));
        } else if (d->T > kSteps) {
            PPO_TRY((pass<T, NL, MARKS>(a, two, 1, st)));
        }
        PPO_TRY((vec ? back_launch<T, 8 * NL, true>(a, st) : back_launch<T, 8 * NL, false>(a, st)));
        const long long few = (long long)d->T * d->Be * d->groups * 2 * p.NP;
        return ppo_launch(scan_few_kernel<T, 16 * NL>, dim3((unsigned)((few + 255) / 256)), dim3(256), 0, st, a);
    }));
    return params ? ppo_param_sum(a.part, p.parts, {{dA, dD, ddt_bias}, {(long long)d->channels * d->N, d->channels, d->channels}}, accumulate, st) : PPO_OK;
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
            constexpr size_t smem = kAhead * 4 * 256 * sizeof(float4);
            static PerDevice<bool> allowed;
            PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(scan_step_kernel<T, NL>, smem); }));
            // as many envs a block as make one round of three blocks an SM
            const int cols = d->groups * ppo_cdiv(d->channels / d->groups, 4 * (256 / NL)), slices = cols < 3 * 148 ? 3 * 148 / cols : 1, envs = ppo_cdiv(d->Be, slices);
            const long long blocks = (long long)cols * ppo_cdiv(d->Be, envs);
            if (blocks > 0x7fffffffll) return PPO_ERR_UNSUPPORTED;
            return ppo_launch(scan_step_kernel<T, NL>, dim3((unsigned)blocks), dim3(256), smem, static_cast<cudaStream_t>(stream), a, envs);
        };
        if (d->N <= 4) return run(std::integral_constant<int, 1>{});
        if (d->N <= 8) return run(std::integral_constant<int, 2>{});
        if (d->N <= 16) return run(std::integral_constant<int, 4>{});
        if (d->N <= 32) return run(std::integral_constant<int, 8>{});
        return run(std::integral_constant<int, 16>{});
    });
}
