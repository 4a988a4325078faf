// Group normalisation with an activation, channels last, and its gradients.
//
// Means, squares about the mean and all arithmetic in 32 bits (variances never as a difference of squares); what is stored is rounded
// once.  Read once, written once where an image, or its group, fits registers or the shared memory of a cluster.
#include "elem.cuh"
#include "tcgen05.cuh"

namespace {

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    float *mean, *rstd;
    float *part;  // shares of the gradients of gamma and beta, [parts][2][C]
    long long ldx, ldy;
    int B, HW, C, groups, per;
    float eps;
};

// kBlocks: an image is split over 1, 2, 4 or 8 blocks until an SM has shared memory for at least so many.  1024 images of 1200 x 64, bf16: 2
// (2 blocks an image) 85 us; 3, 4 or 5 (4 blocks an image, of which an SM holds five) 79; 6 (8 blocks an image) 116.
constexpr int kThreads = 256, kBlocks = 3;

// Sum over the block, the same in every thread; tmp holds one value per warp.
__device__ __forceinline__ float block_sum(float v, float *tmp) {
    v = warp_sum(v);
    __syncthreads();
    if (threadIdx.x % 32 == 0) tmp[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < kThreads / 32; ++i) v += tmp[i];
    return v;
}
// Sum over `lanes` (a power of two) neighbouring lanes, the same in each.
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float activate(float z) {
    return ACT == PPO_ACT_RELU ? (z < 0.f ? 0.f : z) : ACT == PPO_ACT_SILU ? z * sigmoid(z) : z;
}

// z = gamma xhat + beta as one product: (x - mean) scale + shift with scale = rstd gamma, shift = beta.
struct Affine {
    float scale, shift;
};

// Out of line: its 64-bit registers are no part of the kernels' own.
__device__ __noinline__ bool open_exactly(float x, float mean, float rstd, float gamma, float shift) {
    return ((double)x - (double)mean) * (double)rstd * (double)gamma + (double)shift > 0.;
}

// dL/dz.  Which side of 0 z is on decides the ReLU's gradient; 32 bits decide it wrongly only where the two terms of z cancel to
// within their own rounding (three units of the last place of the product), and there 64 bits do.
template <int ACT>
__device__ __forceinline__ float grad_z(float dy, float xc, Affine f, float x, float mean, float rstd, float gamma) {
    if (ACT == PPO_ACT_NONE) return dy;
    const float z = fmaf(xc, f.scale, f.shift);
    if (ACT == PPO_ACT_SILU) {
        const float p = sigmoid(z);
        return dy * (p * fmaf(z, 1.f - p, 1.f));
    }
    bool open = z > 0.f;
    if (fabsf(z) <= 5e-7f * fabsf(f.shift)) open = open_exactly(x, mean, rstd, gamma, f.shift);
    return open ? dy : 0.f;
}

// dL/dz of a vector: gated for the ReLU.  xc = x - mean, per element; the check for values next to 0 is one for all of them.
template <int ACT, int N, int M>
__device__ __forceinline__ void grad_vector(float (&e)[N], const float (&xc)[N], const float (&x)[N], const float (&mean)[N / M], const float (&rstd)[N / M],
                                            const float *gamma, const float (&scale)[N], const float (&beta)[N]) {
    if constexpr (ACT == PPO_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float z = fmaf(xc[k], scale[k], beta[k]), p = sigmoid(z);
            e[k] *= p * fmaf(z, 1.f - p, 1.f);
        }
    } else if constexpr (ACT == PPO_ACT_RELU) {
        bool near = false;
        float z[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            z[k] = fmaf(xc[k], scale[k], beta[k]);
            near |= fabsf(z[k]) <= 5e-7f * fabsf(beta[k]);
        }
        if (near) {
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = grad_z<ACT>(e[k], xc[k], {scale[k], beta[k]}, x[k], mean[k / M], rstd[k / M], gamma ? gamma[k] : 1.f);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) e[k] = z[k] > 0.f ? e[k] : 0.f;
        }
    }
}

// ---- any channel count, stride and alignment: a block per image and group, element by element ----

// Threads (p, c): c channels of the group side by side, p pixels.
struct Tile {
    int lanes, rows, c, p;
    __device__ Tile(int per) {
        lanes = min(per, kThreads);
        rows = kThreads / lanes;
        c = threadIdx.x % lanes;
        p = threadIdx.x / lanes;
    }
};

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) norm_fwd_any_kernel(NormArgs a) {
    grid_wait();
    __shared__ float tmp[kThreads / 32];
    const int b = blockIdx.x / a.groups, g = blockIdx.x % a.groups, c0 = g * a.per;
    const T *x = static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0;
    T *y = static_cast<T *>(a.y) + (long long)b * a.HW * a.ldy + c0;
    const float n = (float)a.HW * (float)a.per;
    const Tile t(a.per);
    float s = 0.f;
    if (t.p < t.rows)
        for (int c = t.c; c < a.per; c += t.lanes)
            for (int i = t.p; i < a.HW; i += t.rows) s += to_f32(x[i * a.ldx + c]);
    const float mean = block_sum(s, tmp) / n;
    s = 0.f;
    if (t.p < t.rows)
        for (int c = t.c; c < a.per; c += t.lanes)
            for (int i = t.p; i < a.HW; i += t.rows) {
                const float d = to_f32(x[i * a.ldx + c]) - mean;
                s = fmaf(d, d, s);
            }
    const float rstd = 1.f / sqrtf(block_sum(s, tmp) / n + a.eps);
    if (threadIdx.x == 0) {
        a.mean[blockIdx.x] = mean;
        a.rstd[blockIdx.x] = rstd;
    }
    if (t.p < t.rows)
        for (int c = t.c; c < a.per; c += t.lanes) {
            const float scale = rstd * (a.gamma ? a.gamma[c0 + c] : 1.f), shift = a.gamma ? a.beta[c0 + c] : 0.f;
            for (int i = t.p; i < a.HW; i += t.rows) y[i * a.ldy + c] = from_f32<T>(activate<ACT>(fmaf(to_f32(x[i * a.ldx + c]) - mean, scale, shift)));
        }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) norm_bwd_any_kernel(NormArgs a) {
    grid_wait();
    __shared__ float tmp[kThreads / 32], part[2][kThreads];
    const int b = blockIdx.x / a.groups, g = blockIdx.x % a.groups, c0 = g * a.per;
    const T *x = static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0, *dy = static_cast<const T *>(a.dy) + (long long)b * a.HW * a.ldy + c0;
    T *dx = static_cast<T *>(a.dx) + (long long)b * a.HW * a.ldx + c0;
    const float mean = a.mean[blockIdx.x], rstd = a.rstd[blockIdx.x], n = (float)a.HW * (float)a.per;
    const Tile t(a.per);
    float m1 = 0.f, m2 = 0.f;
    for (int c = t.c; c - t.c < a.per; c += t.lanes) {
        const bool on = c < a.per && t.p < t.rows;
        const float gamma = on && a.gamma ? a.gamma[c0 + c] : 1.f;
        const Affine f = {rstd * gamma, on && a.gamma ? a.beta[c0 + c] : 0.f};
        float s1 = 0.f, s2 = 0.f;
        if (on)
            for (int i = t.p; i < a.HW; i += t.rows) {
                const float v = to_f32(x[i * a.ldx + c]), xc = v - mean, dz = grad_z<ACT>(to_f32(dy[i * a.ldy + c]), xc, f, v, mean, rstd, gamma);
                s1 += dz;
                s2 = fmaf(dz, xc, s2);
            }
        __syncthreads();
        part[0][threadIdx.x] = s1;
        part[1][threadIdx.x] = s2;
        __syncthreads();
        if (t.p == 0 && on) {
            for (int p = 1; p < t.rows; ++p) {
                s1 += part[0][p * t.lanes + t.c];
                s2 += part[1][p * t.lanes + t.c];
            }
            s2 *= rstd;
            if (a.part) {
                a.part[(size_t)b * 2 * a.C + c0 + c] = s2;
                a.part[((size_t)b * 2 + 1) * a.C + c0 + c] = s1;
            }
            m1 = fmaf(gamma, s1, m1);
            m2 = fmaf(gamma, s2, m2);
        }
    }
    m1 = block_sum(m1, tmp) / n;
    m2 = block_sum(m2, tmp) / n * rstd;
    if (t.p < t.rows)
        for (int c = t.c; c < a.per; c += t.lanes) {
            const float gamma = a.gamma ? a.gamma[c0 + c] : 1.f;
            const Affine f = {rstd * gamma, a.gamma ? a.beta[c0 + c] : 0.f};
            for (int i = t.p; i < a.HW; i += t.rows) {
                const float v = to_f32(x[i * a.ldx + c]), xc = v - mean, dz = grad_z<ACT>(to_f32(dy[i * a.ldy + c]), xc, f, v, mean, rstd, gamma);
                dx[i * a.ldx + c] = from_f32<T>(rstd * (fmaf(gamma, dz, -m1) - xc * m2));
            }
        }
}

// ---- few values per image and group (up to 256 vectors): `width` lanes of a warp per group, its values in registers ----
//
// `active` of them, a multiple of a pixel's vectors of the group: a lane's vectors hold the same channels at every pixel, so it keeps
// their scales, and the sums over images of their gradients, for all images its block goes through.  Gradients of 4096 rows of 1024 in 16
// groups, fp32: 18.6 us with the sum of the shares, whose launch is a third of it (element by element 4094; 2 x 148 blocks 23.3).

struct Lanes {
    int width, active;
};

template <typename T, int ACT, int NV>
__global__ void __launch_bounds__(kThreads) norm_fwd_small_kernel(NormArgs a, Lanes ln, int items) {
    grid_wait();
    constexpr int N = Vec<T>::N;
    const int vecs = a.per / N, all = a.HW * vecs, l = threadIdx.x % ln.width;
    const unsigned item = blockIdx.x * (kThreads / ln.width) + threadIdx.x / ln.width;
    const bool on = item < (unsigned)items && l < ln.active;
    const int b = on ? (int)(item / a.groups) : 0, g = on ? (int)(item % a.groups) : 0, c0 = g * a.per + l % vecs * N;
    const T *x = static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0;
    Vec<T> v[NV];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = i * ln.active + l;
        v[i].raw = on && at < all ? *reinterpret_cast<const uint4 *>(x + at / vecs * a.ldx) : make_uint4(0, 0, 0, 0);
    }
    const float n = (float)a.HW * (float)a.per;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float f[N];
        v[i].get(f);
#pragma unroll
        for (int k = 0; k < N; ++k) s += f[k];
    }
    const float mean = lanes_sum(s, ln.width) / n;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float f[N];
        v[i].get(f);
        if (on && i * ln.active + l < all) {
#pragma unroll
            for (int k = 0; k < N; ++k) s = fmaf(f[k] - mean, f[k] - mean, s);
        }
    }
    const float rstd = 1.f / sqrtf(lanes_sum(s, ln.width) / n + a.eps);
    if (!on) return;
    if (l == 0) {
        a.mean[item] = mean;
        a.rstd[item] = rstd;
    }
    float scale[N], shift[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        scale[k] = a.gamma ? rstd * a.gamma[c0 + k] : rstd;
        shift[k] = a.gamma ? a.beta[c0 + k] : 0.f;
    }
    T *y = static_cast<T *>(a.y) + (long long)b * a.HW * a.ldy + c0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = i * ln.active + l;
        float f[N];
        v[i].get(f);
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = activate<ACT>(fmaf(f[k] - mean, scale[k], shift[k]));
        v[i].set(f);
        if (at < all) *reinterpret_cast<uint4 *>(y + at / vecs * a.ldy) = v[i].raw;
    }
}

// Block (x, y): groups y * kThreads / width .. of the images x, x + gridDim.x, ...  From NV = 4 on the values are read again (from L1)
// instead of kept.
template <typename T, int ACT, int NV>
__global__ void __launch_bounds__(kThreads, 2) norm_bwd_small_kernel(NormArgs a, Lanes ln) {
    grid_wait();
    constexpr int N = Vec<T>::N, KEEP = NV < 4 ? NV : 1;
    const int vecs = a.per / N, all = a.HW * vecs, l = threadIdx.x % ln.width;
    const int g = blockIdx.y * (kThreads / ln.width) + threadIdx.x / ln.width;
    const bool on = g < a.groups && l < ln.active;
    const int c0 = (on ? g * a.per : 0) + l % vecs * N;
    const float n = (float)a.HW * (float)a.per;
    float gamma[N], beta[N], s1[N], s2[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        gamma[k] = a.gamma ? a.gamma[c0 + k] : 1.f;
        beta[k] = a.gamma ? a.beta[c0 + k] : 0.f;
        s1[k] = s2[k] = 0.f;
    }
    struct Image {
        float mean[1], rstd[1];
        Vec<T> v[KEEP], d[KEEP];
    };
    const auto load = [&](int b, int i, Vec<T> &vx, Vec<T> &vd) {
        const int at = i * ln.active + l, p = at / vecs;
        const bool ok = on && at < all && b < a.B;
        const T *x = static_cast<const T *>(a.x) + (long long)b * a.HW * a.ldx + c0, *dy = static_cast<const T *>(a.dy) + (long long)b * a.HW * a.ldy + c0;
        vx.raw = ok ? *reinterpret_cast<const uint4 *>(x + p * a.ldx) : make_uint4(0, 0, 0, 0);
        vd.raw = ok ? *reinterpret_cast<const uint4 *>(dy + p * a.ldy) : make_uint4(0, 0, 0, 0);
    };
    const auto fetch = [&](int b, Image &m) {
        const bool ok = on && b < a.B;
        m.mean[0] = ok ? a.mean[(long long)b * a.groups + g] : 0.f;
        m.rstd[0] = ok ? a.rstd[(long long)b * a.groups + g] : 0.f;
        if constexpr (KEEP == NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load(b, i, m.v[i], m.d[i]);
        }
    };
    const auto work = [&](int b, Image &m) {
        T *dx = static_cast<T *>(a.dx) + (long long)b * a.HW * a.ldx + c0;
        const float rstd = m.rstd[0];
        float scale[N];
#pragma unroll
        for (int k = 0; k < N; ++k) scale[k] = rstd * gamma[k];
        const auto both = [&](const Vec<T> &vx, const Vec<T> &vd, float (&xc)[N], float (&dz)[N]) {
            float f[N];
            vx.get(f);
            vd.get(dz);
#pragma unroll
            for (int k = 0; k < N; ++k) xc[k] = f[k] - m.mean[0];
            grad_vector<ACT, N, N>(dz, xc, f, m.mean, m.rstd, a.gamma ? a.gamma + c0 : nullptr, scale, beta);
        };
        float m1 = 0.f, m2 = 0.f;
#pragma unroll(KEEP == NV ? NV : 2)
        for (int i = 0; i < NV; ++i) {
            if constexpr (KEEP != NV) load(b, i, m.v[0], m.d[0]);
            float xc[N], dz[N];
            both(m.v[i % KEEP], m.d[i % KEEP], xc, dz);
            if (on && i * ln.active + l < all) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    s1[k] += dz[k];
                    s2[k] = fmaf(dz[k], xc[k] * rstd, s2[k]);
                    m1 = fmaf(gamma[k], dz[k], m1);
                    m2 = fmaf(gamma[k] * dz[k], xc[k], m2);
                }
            }
        }
        m1 = lanes_sum(m1, ln.width) / n;
        m2 = lanes_sum(m2, ln.width) / n * rstd * rstd;
#pragma unroll(KEEP == NV ? NV : 2)
        for (int i = 0; i < NV; ++i) {
            if constexpr (KEEP != NV) load(b, i, m.v[0], m.d[0]);
            const int at = i * ln.active + l;
            float xc[N], dz[N];
            both(m.v[i % KEEP], m.d[i % KEEP], xc, dz);
#pragma unroll
            for (int k = 0; k < N; ++k) dz[k] = rstd * (fmaf(gamma[k], dz[k], -m1) - xc[k] * m2);
            Vec<T> r;
            r.set(dz);
            if (on && at < all) *reinterpret_cast<uint4 *>(dx + at / vecs * a.ldx) = r.raw;
        }
    };
    constexpr int AT_ONCE = KEEP == NV ? 2 : 1;  // images whose loads are on their way (38907 rows of 32 x 24 bf16: 169 us by one, 142)
    for (int b = blockIdx.x; b < a.B; b += AT_ONCE * gridDim.x) {
        Image image[AT_ONCE];
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) fetch(b + q * (int)gridDim.x, image[q]);
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q)
            if (b + q * (int)gridDim.x < a.B) work(b + q * (int)gridDim.x, image[q]);
    }
    if (!a.part) return;
    // lanes of other pixels of the same channels
    const int pixels = ln.active / vecs;
    if ((pixels & (pixels - 1)) == 0 && ln.active == ln.width) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            for (int o = vecs; o < ln.width; o <<= 1) {
                s1[k] += __shfl_xor_sync(0xffffffffu, s1[k], o);
                s2[k] += __shfl_xor_sync(0xffffffffu, s2[k], o);
            }
    } else {  // lane l < vecs adds those of l + vecs, l + 2 vecs, ...
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float t1 = s1[k], t2 = s2[k];
            for (int p = 1; p < pixels; ++p) {
                t1 += __shfl_sync(0xffffffffu, s1[k], l + p * vecs, ln.width);
                t2 += __shfl_sync(0xffffffffu, s2[k], l + p * vecs, ln.width);
            }
            s1[k] = t1;
            s2[k] = t2;
        }
    }
    if (on && l < vecs) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            a.part[(size_t)blockIdx.x * 2 * a.C + c0 + k] = s2[k];
            a.part[((size_t)blockIdx.x * 2 + 1) * a.C + c0 + k] = s1[k];
        }
    }
}

// ---- larger images: several blocks per image, each with a run of its pixels ----
//
// Thread (pl, vc) has the same vector of channels of the pixels pl, pl + lanes, ...: memory is read and written in whole rows.
// K: parts of a vector that belong to different groups (1: a group has whole vectors).
//   WHOLE: a cluster per image, whose blocks keep their pixels in shared memory between the sums, which they exchange there, and
// the result: read once, written once.  What a thread copies in is what it uses, so that only the sums meet at barriers.  1024 x 1200 x 64
// bf16: 79 us, 4.0 TB/s (element by element 449); gradients of 512 x 4800 x 32: 160 us, 3.0 TB/s (814), in clusters of 8 with two blocks on
// an SM: a block loads, sums, meets the others and stores in turn, and only its neighbours on the SM fill the gaps.  The gradients' inputs
// read again from L2 instead of kept: 195 to 247.
//   SUMS, then APPLY: images that do not fit eight blocks; the sums go through the workspace, and the second launch reads the image again.
enum { WHOLE, SUMS, APPLY };

struct Split {
    int n, pixels;  // blocks per image, pixels per block
    size_t smem;
    float *sums;    // SUMS, APPLY: [B][n][groups][2]
};

// Entries of group g among the threads' K parts: thread pl * VC + first + i has part k; pl < lanes, i < span.
struct Members {
    int first, span, k;
};
template <int N, int K>
__device__ __forceinline__ Members members(int g, int per) {
    return K == 1 ? Members{g * (per / N), per / N, 0} : Members{g / K, 1, g % K};
}
// A pair of numbers of this block (rank) and group, to every block of the cluster.
__device__ __forceinline__ void send(float *sent, int rank, int groups, int g, int n, float a, float b) {
    const int to = threadIdx.x % 32;
    if (to < n) {
        const uint32_t at = tc::in_cta(tc::smem_u32(sent + (rank * groups + g) * 2), to);
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(a) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(b) : "memory");
    }
}

template <typename T, int ACT, int K, int MODE>
__global__ void __launch_bounds__(kThreads) norm_fwd_image_kernel(NormArgs a, Split sp) {
    grid_wait();
    if (MODE == WHOLE) tc::cluster_arrive();
    constexpr int N = Vec<T>::N, M = N / K;
    extern __shared__ __align__(16) float mem[];
    float *tm = mem, *tq = tm + kThreads * K, *sent = tq + kThreads * K, *stat = sent + (MODE == WHOLE ? (sp.n * a.groups * 2 + 3) / 4 * 4 : 0);
    uint4 *kept = reinterpret_cast<uint4 *>(stat + (a.groups * 2 + 3) / 4 * 4);
    const int rank = blockIdx.x % sp.n, b = blockIdx.x / sp.n;
    const int VC = a.C / N, lanes = kThreads / VC, tid = threadIdx.x, pl = tid / VC, vc = tid % VC;
    const int p0 = rank * sp.pixels, P = max(0, min(sp.pixels, a.HW - p0));
    const int cnt = pl < lanes && pl < P ? (P - 1 - pl) / lanes + 1 : 0;
    const T *x = static_cast<const T *>(a.x) + ((long long)b * a.HW + p0 + pl) * a.ldx + vc * N;
    T *y = static_cast<T *>(a.y) + ((long long)b * a.HW + p0 + pl) * a.ldy + vc * N;
    const long long sx = lanes * a.ldx, sy = lanes * a.ldy;
    if (MODE == WHOLE) {
        for (int i = 0; i < cnt; ++i) tc::cp_async16(tc::smem_u32(kept + i * kThreads + tid), x + i * sx, true);
        tc::cp_async_commit();
        tc::cp_async_wait<0>();
    }
    const auto get = [&](int i, float (&f)[N]) {
        Vec<T> v;
        v.raw = MODE == WHOLE ? kept[i * kThreads + tid] : *reinterpret_cast<const uint4 *>(x + i * sx);
        v.get(f);
    };
    if constexpr (MODE != APPLY) {
        // mean and squares about it of this thread's values, then of the block's
        float m[K], q[K];
#pragma unroll
        for (int k = 0; k < K; ++k) m[k] = q[k] = 0.f;
#pragma unroll 4
        for (int i = 0; i < cnt; ++i) {
            float f[N];
            get(i, f);
#pragma unroll
            for (int k = 0; k < N; ++k) m[k / M] += f[k];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) m[k] = cnt ? m[k] / (float)(cnt * M) : 0.f;
#pragma unroll 4
        for (int i = 0; i < cnt; ++i) {
            float f[N];
            get(i, f);
#pragma unroll
            for (int k = 0; k < N; ++k) q[k / M] = fmaf(f[k] - m[k / M], f[k] - m[k / M], q[k / M]);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            tm[tid * K + k] = m[k];
            tq[tid * K + k] = q[k];
        }
        __syncthreads();
        if (MODE == WHOLE) tc::cluster_wait();  // all blocks of the cluster run
        for (int g = tid / 32; g < a.groups; g += kThreads / 32) {
            const Members e = members<N, K>(g, a.per);
            const float total = (float)P * (float)a.per;
            float sum = 0.f, sq = 0.f;
            for (int i = tid % 32; i < lanes * e.span; i += 32) {
                const int p = i / e.span, t = p * VC + e.first + i % e.span;
                const float w = p < P ? (float)(((P - 1 - p) / lanes + 1) * M) : 0.f;
                sum = fmaf(w, tm[t * K + e.k], sum);
            }
            const float mean = P ? warp_sum(sum) / total : 0.f;
            for (int i = tid % 32; i < lanes * e.span; i += 32) {
                const int p = i / e.span, t = p * VC + e.first + i % e.span;
                const float w = p < P ? (float)(((P - 1 - p) / lanes + 1) * M) : 0.f, d = tm[t * K + e.k] - mean;
                if (w > 0.f) sq += fmaf(w * d, d, tq[t * K + e.k]);
            }
            sq = warp_sum(sq);
            if (MODE == WHOLE) send(sent, rank, a.groups, g, sp.n, mean, sq);
            else if (tid % 32 == 0) *reinterpret_cast<float2 *>(sp.sums + ((size_t)blockIdx.x * a.groups + g) * 2) = make_float2(mean, sq);
        }
        if (MODE == SUMS) return;
        tc::cluster_sync();
    }
    // of the image
    const float *from = MODE == WHOLE ? sent : sp.sums + (size_t)b * sp.n * a.groups * 2;
    for (int g = tid / 32; g < a.groups; g += kThreads / 32) {
        const float per = (float)a.per, n = (float)a.HW * per;
        float sum = 0.f, sq = 0.f;
        for (int r = tid % 32; r < sp.n; r += 32) sum = fmaf((float)max(0, min(sp.pixels, a.HW - r * sp.pixels)) * per, from[(r * a.groups + g) * 2], sum);
        const float mean = warp_sum(sum) / n;
        for (int r = tid % 32; r < sp.n; r += 32) {
            const float w = (float)max(0, min(sp.pixels, a.HW - r * sp.pixels)) * per, d = from[(r * a.groups + g) * 2] - mean;
            if (w > 0.f) sq += fmaf(w * d, d, from[(r * a.groups + g) * 2 + 1]);
        }
        const float rstd = 1.f / sqrtf(warp_sum(sq) / n + a.eps);
        if (tid % 32 == 0) {
            stat[g * 2] = mean;
            stat[g * 2 + 1] = rstd;
            if (rank == 0) {
                a.mean[(long long)b * a.groups + g] = mean;
                a.rstd[(long long)b * a.groups + g] = rstd;
            }
        }
    }
    __syncthreads();
    if (cnt == 0) return;
    float mean[K], scale[N], shift[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int c = vc * N + k, g = K == 1 ? c / a.per : vc * K + k / M;
        const float rstd = stat[g * 2 + 1];
        mean[k / M] = stat[g * 2];
        scale[k] = a.gamma ? rstd * a.gamma[c] : rstd;
        shift[k] = a.gamma ? a.beta[c] : 0.f;
    }
#pragma unroll 4
    for (int i = 0; i < cnt; ++i) {
        float f[N];
        get(i, f);
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = activate<ACT>(fmaf(f[k] - mean[k / M], scale[k], shift[k]));
        Vec<T> v;
        v.set(f);
        *reinterpret_cast<uint4 *>(y + i * sy) = v.raw;
    }
}

template <typename T, int ACT, int K, int MODE>
__global__ void __launch_bounds__(kThreads, 3) norm_bwd_image_kernel(NormArgs a, Split sp) {
    grid_wait();
    if (MODE == WHOLE) tc::cluster_arrive();
    constexpr int N = Vec<T>::N, M = N / K;
    extern __shared__ __align__(16) float mem[];
    constexpr int kPitch = kThreads + 1;  // of a sum's shares: no eight of one bank
    float *ts = mem, *chan = ts + (kPitch * 2 * N + 3) / 4 * 4, *sent = chan + 2 * a.C, *stat = sent + (MODE == WHOLE ? (sp.n * a.groups * 2 + 3) / 4 * 4 : 0);
    uint4 *keptx = reinterpret_cast<uint4 *>(stat + (a.groups * 2 + 3) / 4 * 4);
    const int rank = blockIdx.x % sp.n, b = blockIdx.x / sp.n;
    const int VC = a.C / N, lanes = kThreads / VC, tid = threadIdx.x, pl = tid / VC, vc = tid % VC;
    const int p0 = rank * sp.pixels, P = max(0, min(sp.pixels, a.HW - p0)), rounds = (sp.pixels + lanes - 1) / lanes;
    uint4 *keptd = keptx + rounds * kThreads;
    const int cnt = pl < lanes && pl < P ? (P - 1 - pl) / lanes + 1 : 0;
    const long long px = ((long long)b * a.HW + p0 + pl) * a.ldx + vc * N, py = ((long long)b * a.HW + p0 + pl) * a.ldy + vc * N;
    const T *x = static_cast<const T *>(a.x) + px, *dy = static_cast<const T *>(a.dy) + py;
    T *dx = static_cast<T *>(a.dx) + px;
    const long long sx = lanes * a.ldx, sy = lanes * a.ldy;
    if (MODE == WHOLE) {
        for (int i = 0; i < cnt; ++i) {
            tc::cp_async16(tc::smem_u32(keptx + i * kThreads + tid), x + i * sx, true);
            tc::cp_async16(tc::smem_u32(keptd + i * kThreads + tid), dy + i * sy, true);
        }
        tc::cp_async_commit();
    }
    float mean[K], rstd[K], scale[N], beta[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int c = min(vc * N + k, a.C - 1), g = K == 1 ? c / a.per : vc * K + k / M;
        mean[k / M] = a.mean[(long long)b * a.groups + g];
        rstd[k / M] = a.rstd[(long long)b * a.groups + g];
        beta[k] = a.gamma ? a.beta[c] : 0.f;
        scale[k] = a.gamma ? rstd[k / M] * a.gamma[c] : rstd[k / M];
    }
    if (MODE == WHOLE) tc::cp_async_wait<0>();
    // x - mean and dL/dz; a gated dL/dy of the ReLU is kept, in the place of dL/dy, for the second time
    const auto get = [&](int i, float (&xc)[N], float (&dz)[N], bool again) {
        Vec<T> v, d;
        v.raw = MODE == WHOLE ? keptx[i * kThreads + tid] : *reinterpret_cast<const uint4 *>(x + i * sx);
        d.raw = MODE == WHOLE ? keptd[i * kThreads + tid] : *reinterpret_cast<const uint4 *>(dy + i * sy);
        float f[N];
        v.get(f);
        d.get(dz);
#pragma unroll
        for (int k = 0; k < N; ++k) xc[k] = f[k] - mean[k / M];
        if (MODE == WHOLE && ACT == PPO_ACT_RELU && again) return;
        grad_vector<ACT, N, M>(dz, xc, f, mean, rstd, a.gamma ? a.gamma + vc * N : nullptr, scale, beta);
        if (MODE == WHOLE && ACT == PPO_ACT_RELU) {
            d.set(dz);
            keptd[i * kThreads + tid] = d.raw;
        }
    };
    if constexpr (MODE != APPLY) {
        float s1[N], s2[N];
#pragma unroll
        for (int k = 0; k < N; ++k) s1[k] = s2[k] = 0.f;
#pragma unroll 2
        for (int i = 0; i < cnt; ++i) {
            float xc[N], dz[N];
            get(i, xc, dz, false);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                s1[k] += dz[k];
                s2[k] = fmaf(dz[k], xc[k], s2[k]);
            }
        }
        // [2][N][threads]
#pragma unroll
        for (int k = 0; k < N; ++k) {
            ts[k * kPitch + tid] = s1[k];
            ts[(N + k) * kPitch + tid] = s2[k] * rstd[k / M];
        }
        __syncthreads();
        if (MODE == WHOLE) tc::cluster_wait();  // all blocks of the cluster run
        int sub = 1;  // lanes per channel and sum
        while (sub < 32 && sub * 2 * 2 * a.C <= kThreads) sub *= 2;
        for (int i0 = 0; i0 < 2 * a.C; i0 += kThreads / sub) {
            const int i = i0 + tid / sub, k2 = i / a.C, c = i % a.C;
            float s = 0.f;
            if (i < 2 * a.C)
                for (int p = tid % sub; p < lanes; p += sub) s += ts[(k2 * N + c % N) * kPitch + p * VC + c / N];
            s = lanes_sum(s, sub);
            if (i < 2 * a.C && tid % sub == 0) {
                chan[i] = s;
                if (a.part) a.part[((size_t)blockIdx.x * 2 + 1 - k2) * a.C + c] = s;  // gamma's first
            }
        }
        __syncthreads();
        for (int g = tid / 32; g < a.groups; g += kThreads / 32) {
            float m1 = 0.f, m2 = 0.f;
            for (int c = g * a.per + tid % 32; c < (g + 1) * a.per; c += 32) {
                const float w = a.gamma ? a.gamma[c] : 1.f;
                m1 = fmaf(w, chan[c], m1);
                m2 = fmaf(w, chan[a.C + c], m2);
            }
            m1 = warp_sum(m1);
            m2 = warp_sum(m2);
            if (MODE == WHOLE) send(sent, rank, a.groups, g, sp.n, m1, m2);
            else if (tid % 32 == 0) *reinterpret_cast<float2 *>(sp.sums + ((size_t)blockIdx.x * a.groups + g) * 2) = make_float2(m1, m2);
        }
        if (MODE == SUMS) return;
        tc::cluster_sync();
    }
    const float *from = MODE == WHOLE ? sent : sp.sums + (size_t)b * sp.n * a.groups * 2;
    for (int g = tid / 32; g < a.groups; g += kThreads / 32) {
        float m1 = 0.f, m2 = 0.f;
        for (int r = tid % 32; r < sp.n; r += 32) {
            m1 += from[(r * a.groups + g) * 2];
            m2 += from[(r * a.groups + g) * 2 + 1];
        }
        const float n = (float)a.HW * (float)a.per;
        m1 = warp_sum(m1);
        m2 = warp_sum(m2);
        if (tid % 32 == 0) {
            stat[g * 2] = m1 / n;
            stat[g * 2 + 1] = m2 / n;
        }
    }
    __syncthreads();
    if (cnt == 0) return;
    // dx = scale dz + (D xc + E)
    float D[K], E[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int g = K == 1 ? vc * N / a.per : vc * K + k;
        D[k] = -rstd[k] * rstd[k] * stat[g * 2 + 1];
        E[k] = -rstd[k] * stat[g * 2];
    }
#pragma unroll 2
    for (int i = 0; i < cnt; ++i) {
        float xc[N], dz[N];
        get(i, xc, dz, true);
#pragma unroll
        for (int k = 0; k < N; ++k) dz[k] = fmaf(scale[k], dz[k], fmaf(D[k / M], xc[k], E[k / M]));
        Vec<T> v;
        v.set(dz);
        *reinterpret_cast<uint4 *>(dx + i * sx) = v.raw;
    }
}

// Sums of the shares, in a fixed order: 32 channels per cluster of n blocks, 16 warps each with every 16 n-th share.
__global__ void __launch_bounds__(512) norm_sum_kernel(const float *part, int parts, int C, float *dgamma, float *dbeta, int accumulate, int n) {
    grid_wait();
    if (n > 1) tc::cluster_arrive();
    __shared__ double sum[16][33], whole[8][32];
    const int rank = blockIdx.x % n, l = threadIdx.x % 32, c = blockIdx.x / n * 32 + l, w = threadIdx.x / 32, k = blockIdx.y;
    double s = 0;
    if (c < C) {
#pragma unroll 8
        for (int i = rank * 16 + w; i < parts; i += 16 * n) s += part[((size_t)i * 2 + k) * C + c];
    }
    sum[w][l] = s;
    __syncthreads();
    if (n > 1) tc::cluster_wait();
    if (w == 0) {
        for (int i = 1; i < 16; ++i) s += sum[i][l];
        if (n > 1) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(tc::in_cta(tc::smem_u32(&whole[rank][l]), 0)), "d"(s) : "memory");
    }
    if (n > 1) {
        tc::cluster_sync();
        if (rank == 0 && w == 0) {
            s = whole[0][l];
            for (int i = 1; i < n; ++i) s += whole[i][l];
        }
    }
    if (rank == 0 && w == 0 && c < C) {
        float *out = k == 0 ? dgamma : dbeta;
        out[c] = (float)(s + (accumulate ? (double)out[c] : 0.));
    }
}

// ---- which kernel ----

struct Plan {
    enum { ANY, SMALL, IMAGE } kind;
    Lanes lanes;     // SMALL: per group; vectors per lane, blocks along the images (backward)
    int nv, blocks;
    int K, whole;    // IMAGE
    Split sp;
    int parts;       // shares of the gradients of gamma and beta
    size_t floats;   // of the workspace
};

// By sizes alone (so that the workspace is known before the addresses are); rows that turn out not to be aligned take the kernels
// for any alignment, whose shares (one per image) fit in the same workspace.
Plan plan_of(const ppo_group_norm_desc *d, bool bwd) {
    Plan p = {};
    const int size = (int)elem_bytes(d->dtype), N = 16 / size, per = d->C / d->groups;
    p.kind = Plan::ANY;
    p.parts = d->B;
    p.floats = bwd ? (size_t)2 * d->B * d->C : 0;
    if (d->C % N != 0 || d->ldx % N != 0 || d->ldy % N != 0) return p;
    const long long all = (long long)d->HW * per / N;  // vectors of an image and group
    const int vecs = per / N;
    p.K = per % N == 0 ? 1 : N % per == 0 ? N / per : 0;
    const int VC = d->C / N;
    const bool image = p.K != 0 && VC <= kThreads && d->groups <= 1024;
    // gradients that a lane does not keep are left to the blocks of an image: 2048 images of 32 x 256 in 4 groups, bf16, 58 and 87 us, of
    // 16 x 256 50 and 52, of 8 x 256 77 and 38 (kept); outputs 41 and 29, 35 and 18, 55 and 18
    const int most = bwd && image ? 4 : 8;
    if (per % N == 0 && vecs <= 32 && all <= 32 / vecs * vecs * most) {
        int width = 1;  // as few lanes as hold the group in a vector each (38907 rows of 32 x 24 bf16: 672 us by whole warps, now 142)
        while (width < vecs || (width < 32 && width / vecs * vecs < all)) width *= 2;
        const int active = width / vecs * vecs;
        p.kind = Plan::SMALL;
        p.lanes = {width, active};
        p.nv = all <= active ? 1 : all <= 2 * active ? 2 : all <= 4 * active ? 4 : 8;
        const int columns = ppo_cdiv(d->groups, kThreads / width);
        if (bwd && columns > 65535) {  // more than a grid has along y
            p.kind = Plan::ANY;
            return p;
        }
        p.blocks = ppo_cdiv(4 * 148, columns);
        if (p.blocks > d->B) p.blocks = d->B;
        p.parts = p.blocks;
    } else {
        if (!image) return p;
        p.kind = Plan::IMAGE;
        const int lanes = kThreads / VC;
        const auto smem = [&](int n, bool whole) {
            const int rounds = ppo_cdiv(ppo_cdiv(d->HW, n), lanes);
            const size_t floats = (bwd ? ((kThreads + 1) * 2 * N + 3) / 4 * 4 + 2 * d->C : kThreads * p.K * 2) + (whole ? ((size_t)n * d->groups * 2 + 3) / 4 * 4 : 0) +
                                  (d->groups * 2 + 3) / 4 * 4;
            return floats * 4 + (whole ? (size_t)rounds * kThreads * 16 * (bwd ? 2 : 1) : 0);
        };
        // as few blocks per image as leave room for kBlocks on an SM, else for two or one
        int n = 1;
        while (n < 8 && smem(n, true) > 227 * 1024 / kBlocks - 1024) n *= 2;
        p.whole = smem(n, true) <= 227 * 1024;
        if (!p.whole) {  // as many as give every SM four, none with less than four rows of its lanes
            n = ppo_cdiv(4 * 148, d->B);
            const int most = ppo_cdiv(d->HW, 4 * lanes);
            if (n > most) n = most;
        }
        p.sp = {n, ppo_cdiv(d->HW, n), smem(n, p.whole), nullptr};
        p.parts = d->B * n;
    }
    p.floats = bwd ? (size_t)2 * (p.parts > d->B ? p.parts : d->B) * d->C : 0;
    if (p.kind == Plan::IMAGE && !p.whole) p.floats += (p.floats & 1) + (size_t)p.parts * d->groups * 2;
    return p;
}

template <typename T, typename F>
int with_act(int act, F &&fn) {
    if (act == PPO_ACT_RELU) return fn(T{}, std::integral_constant<int, PPO_ACT_RELU>{});
    if (act == PPO_ACT_SILU) return fn(T{}, std::integral_constant<int, PPO_ACT_SILU>{});
    return fn(T{}, std::integral_constant<int, PPO_ACT_NONE>{});
}
template <typename F>
int with_elem_act(int dtype, int act, F &&fn) {
    if (dtype == PPO_F32) return with_act<float>(act, fn);
    if (dtype == PPO_BF16) return with_act<bf16>(act, fn);
    return with_act<__half>(act, fn);
}

template <auto FN>
int launch_image(bool cluster, const NormArgs &a, const Split &sp, cudaStream_t st) {
    static PerDevice<bool> allowed;
    PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(FN, 227 * 1024); }));
    const dim3 grid((unsigned)(a.B * sp.n)), block(kThreads);
    return cluster ? ppo_launch_cluster(FN, sp.n, grid, block, sp.smem, st, a, sp) : ppo_launch(FN, grid, block, sp.smem, st, a, sp);
}
template <typename T, int ACT, int K>
int fwd_image(const Plan &p, const NormArgs &a, cudaStream_t st) {
    if (p.whole) return launch_image<norm_fwd_image_kernel<T, ACT, K, WHOLE>>(true, a, p.sp, st);
    PPO_TRY((launch_image<norm_fwd_image_kernel<T, PPO_ACT_NONE, K, SUMS>>(false, a, p.sp, st)));
    return launch_image<norm_fwd_image_kernel<T, ACT, K, APPLY>>(false, a, p.sp, st);
}
template <typename T, int ACT, int K>
int bwd_image(const Plan &p, const NormArgs &a, cudaStream_t st) {
    if (p.whole) return launch_image<norm_bwd_image_kernel<T, ACT, K, WHOLE>>(true, a, p.sp, st);
    PPO_TRY((launch_image<norm_bwd_image_kernel<T, ACT, K, SUMS>>(false, a, p.sp, st)));
    return launch_image<norm_bwd_image_kernel<T, ACT, K, APPLY>>(false, a, p.sp, st);
}

int check(const ppo_group_norm_desc *d) {
    if (!d || d->B <= 0 || d->HW <= 0 || d->C <= 0 || d->groups <= 0) return PPO_ERR_INVALID_ARG;
    if (d->act < PPO_ACT_NONE || d->act > PPO_ACT_SILU || d->dtype < PPO_F32 || d->dtype > PPO_F16) return PPO_ERR_INVALID_ARG;
    if (d->C % d->groups != 0 || d->ldx < d->C || d->ldy < d->C) return PPO_ERR_SHAPE;
    if ((long long)d->B * d->groups > 0x7fffffffll || d->B > 0x0fffffff) return PPO_ERR_UNSUPPORTED;
    return PPO_OK;
}

NormArgs args(const ppo_group_norm_desc *d) {
    NormArgs a = {};
    a.ldx = d->ldx;
    a.ldy = d->ldy;
    a.B = d->B;
    a.HW = d->HW;
    a.C = d->C;
    a.groups = d->groups;
    a.per = d->C / d->groups;
    return a;
}

}  // namespace

extern "C" size_t ppo_group_norm_workspace_bytes(const ppo_group_norm_desc *d, int backward) {
    return check(d) == PPO_OK ? plan_of(d, backward != 0).floats * sizeof(float) : 0;
}

extern "C" int ppo_group_norm_fwd(const ppo_group_norm_desc *d, float eps, const void *x, const float *gamma, const float *beta, void *y, float *mean,
                                  float *rstd, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    if (!x || !y || !mean || !rstd || !gamma != !beta || !(eps >= 0.f)) return PPO_ERR_INVALID_ARG;
    if (x == y && d->ldx != d->ldy) return PPO_ERR_SHAPE;
    const size_t need = ppo_group_norm_workspace_bytes(d, 0), e = elem_bytes(d->dtype);
    if (need > 0 && !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd})
        if (!ppo_aligned(p, 4)) return PPO_ERR_ALIGN;
    if (!ppo_aligned(x, e) || !ppo_aligned(y, e) || !ppo_aligned(workspace, 32)) return PPO_ERR_ALIGN;
    NormArgs a = args(d);
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = eps;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Plan p = plan_of(d, false);
    p.sp.sums = static_cast<float *>(workspace);
    if (!ppo_aligned(x, 16) || !ppo_aligned(y, 16)) p.kind = Plan::ANY;
    return with_elem_act(d->dtype, d->act, [&](auto t, auto act) -> int {
        using T = decltype(t);
        constexpr int ACT = decltype(act)::value, N = Vec<T>::N;
        const dim3 block(kThreads);
        const int items = a.B * a.groups;
        if (p.kind == Plan::ANY) return ppo_launch(norm_fwd_any_kernel<T, ACT>, dim3(items), block, 0, st, a);
        if (p.kind == Plan::SMALL) {
            const dim3 grid(ppo_cdiv(items, kThreads / p.lanes.width));
            if (p.nv == 1) return ppo_launch(norm_fwd_small_kernel<T, ACT, 1>, grid, block, 0, st, a, p.lanes, items);
            if (p.nv == 2) return ppo_launch(norm_fwd_small_kernel<T, ACT, 2>, grid, block, 0, st, a, p.lanes, items);
            if (p.nv == 4) return ppo_launch(norm_fwd_small_kernel<T, ACT, 4>, grid, block, 0, st, a, p.lanes, items);
            return ppo_launch(norm_fwd_small_kernel<T, ACT, 8>, grid, block, 0, st, a, p.lanes, items);
        }
        if (p.K == 1) return fwd_image<T, ACT, 1>(p, a, st);
        if (p.K == 2) return fwd_image<T, ACT, 2>(p, a, st);
        if (p.K == 4) return fwd_image<T, ACT, 4>(p, a, st);
        return fwd_image<T, ACT, N>(p, a, st);
    });
}

extern "C" int ppo_group_norm_bwd(const ppo_group_norm_desc *d, const void *x, const float *gamma, const float *beta, const float *mean,
                                  const float *rstd, const void *dy, void *dx, float *dgamma, float *dbeta, int accumulate, void *workspace,
                                  size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    if (!x || !mean || !rstd || !dy || !dx || !gamma != !beta || !dgamma != !dbeta) return PPO_ERR_INVALID_ARG;
    if (dx == dy && d->ldx != d->ldy) return PPO_ERR_SHAPE;
    const size_t need = ppo_group_norm_workspace_bytes(d, 1), e = elem_bytes(d->dtype);
    if (need > 0 && !workspace) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    for (const void *p : {(const void *)gamma, (const void *)beta, (const void *)mean, (const void *)rstd, (const void *)dgamma, (const void *)dbeta})
        if (!ppo_aligned(p, 4)) return PPO_ERR_ALIGN;
    if (!ppo_aligned(x, e) || !ppo_aligned(dy, e) || !ppo_aligned(dx, e) || !ppo_aligned(workspace, 32)) return PPO_ERR_ALIGN;
    NormArgs a = args(d);
    a.x = x;
    a.dy = dy;
    a.dx = dx;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.part = dgamma ? static_cast<float *>(workspace) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Plan p = plan_of(d, true);
    if (p.kind == Plan::IMAGE && !p.whole) p.sp.sums = static_cast<float *>(workspace) + (p.floats - (size_t)p.parts * d->groups * 2);
    if (!ppo_aligned(x, 16) || !ppo_aligned(dy, 16) || !ppo_aligned(dx, 16)) {
        p.kind = Plan::ANY;
        p.parts = d->B;
    }
    PPO_TRY(with_elem_act(d->dtype, d->act, [&](auto t, auto act) -> int {
        using T = decltype(t);
        constexpr int ACT = decltype(act)::value, N = Vec<T>::N;
        const dim3 block(kThreads);
        if (p.kind == Plan::ANY) return ppo_launch(norm_bwd_any_kernel<T, ACT>, dim3(a.B * a.groups), block, 0, st, a);
        if (p.kind == Plan::SMALL) {
            const dim3 grid(p.blocks, ppo_cdiv(a.groups, kThreads / p.lanes.width));
            if (p.nv == 1) return ppo_launch(norm_bwd_small_kernel<T, ACT, 1>, grid, block, 0, st, a, p.lanes);
            if (p.nv == 2) return ppo_launch(norm_bwd_small_kernel<T, ACT, 2>, grid, block, 0, st, a, p.lanes);
            if (p.nv == 4) return ppo_launch(norm_bwd_small_kernel<T, ACT, 4>, grid, block, 0, st, a, p.lanes);
            return ppo_launch(norm_bwd_small_kernel<T, ACT, 8>, grid, block, 0, st, a, p.lanes);
        }
        if (p.K == 1) return bwd_image<T, ACT, 1>(p, a, st);
        if (p.K == 2) return bwd_image<T, ACT, 2>(p, a, st);
        if (p.K == 4) return bwd_image<T, ACT, 4>(p, a, st);
        return bwd_image<T, ACT, N>(p, a, st);
    }));
    if (!dgamma) return PPO_OK;
    const int n = p.parts > 64 ? 8 : 1, cols = ppo_cdiv(d->C, 32);  // 4096 shares of 32 channels: 80 us by one block, 5 by eight
    const auto sum = [&](auto &&launch) { return launch(dim3(cols * n, 2), dim3(512), 0, st, (const float *)a.part, p.parts, (int)d->C, dgamma, dbeta, accumulate, n); };
    if (n == 1) return sum([&](auto... args) { return ppo_launch(norm_sum_kernel, args...); });
    return sum([&](auto... args) { return ppo_launch_cluster(norm_sum_kernel, n, args...); });
}
