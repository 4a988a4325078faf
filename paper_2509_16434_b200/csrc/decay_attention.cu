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
#include "pair32.cuh"
#include "tcgen05.cuh"
#include "tma_host.cuh"

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
    int seg_len, nseg;   // steps per segment of the sequence (nseg == 1: all); segments are numbered in time's order
    int seg_made;        // 1: an earlier sweep over the same states has left what each segment starts from
    long long seg_r, seg_c;  // strides of a state in it
    float *seg;          // [nseg][Be * heads][R * C]: what each segment adds to a state, then what each starts from
    int *seg_reset;      // [nseg][Be * heads]: whether a done flag is set in it
};

// decay ** n
__device__ __forceinline__ float power(float log2_decay, int n) { return n == 0 ? 1.f : exp2f((float)n * log2_decay); }

// ---- step by step (32 bits, and rows that no vector fits) ----
//
// One block: 64 columns of one head's state over one segment, in registers: two columns a lane, R / 8 rows a warp.  Steps come in tiles of
// 8; a thread fetches its share of the next tile while it works on this one.  Two multiply-adds for each element and step, for two
// rows in one instruction, and a broadcast load of shared memory for sixteen of them: bound by issue and by the chain from step to
// step (gradients of 119 steps of 37 x 6 heads of 48 x 80, fp32: 123 us; one row an instruction 138, one column a lane 183 of two
// launches).  For that the decay is not applied step by step: within a tile the state is kept as N = M lambda^(8-e) behind e steps, so that
// N += a b lambda^(8-e), and out = lambda^(e-8) x^T N.  With lambda >= 1/2 N is at most 2^8 smaller than M, never larger: nothing becomes
// infinite that the formula leaves finite.  Smaller decays are applied step by step, in three operations.  Products of 32-bit numbers have no tensor core instruction without a rounding to 11
// bits; operands as sums of bf16 terms, as the chunks below have them for their states, have not been tried here.
// Sweeps of one call that do not wait for one another, along z of one launch.
struct Sweeps {
    Sweep s[3];
};

constexpr int kTokens = 8, kCols = 64, kSlices = 8;

// STATE: only what the segment leaves behind, from an empty state.
struct StepTiles {
    float a[kTokens * 128], x[kTokens * 128], b[kTokens][kCols], part[kSlices][kTokens][kCols], up[kTokens], down[kTokens + 1];
    int gate[kTokens];
};
template <typename T, int KS, bool STATE>
__device__ __forceinline__ void sweep_rows(const Sweep &s, StepTiles &tile) {
    constexpr int RP = KS * kSlices;
    auto *const ta = reinterpret_cast<float (*)[RP]>(tile.a), *const tx = reinterpret_cast<float (*)[RP]>(tile.x);
    auto &tb = tile.b;
    auto &part = tile.part;
    auto &up = tile.up;
    auto &down = tile.down;
    auto &gate = tile.gate;
    const int tid = threadIdx.x, lane = tid % 32, w = tid / 32;
    const int ncol = (s.C + kCols - 1) / kCols, c0 = blockIdx.x % ncol * kCols;
    const int eh = blockIdx.x / ncol, e = eh / s.heads, h = eh % s.heads;
    const int seg = blockIdx.y, rev = s.reverse;
    const float lam = s.decay[h];
    const bool scaled = lam >= 0.5f;
    const T *A = static_cast<const T *>(s.a) + (long long)(h / s.share_a) * s.R;
    const T *B = static_cast<const T *>(s.b) + (long long)(h / s.share_b) * s.C + c0;
    const T *X = static_cast<const T *>(s.x) + (long long)(h / s.share_x) * s.R;
    if (tid <= kTokens) {
        const float l2 = log2f(lam);
        const int n = kTokens - (tid + 1 - rev);  // decays of a whole tile that come behind step tid
        if (tid < kTokens) up[tid] = scaled ? power(l2, n) : 1.f;
        // what outputs are multiplied with; the last: what the state is in front of a tile
        down[tid] = !scaled ? 1.f : tid < kTokens ? exp2f(-n * l2) : power(l2, kTokens);
    }
    pair32 M[2][KS / 2];  // of two columns, rows in pairs
    // this thread's element of row r of the state lies at r * sr + c * sc
    const long long sr = s.nseg > 1 ? s.seg_r : s.stride_r, sc = s.nseg > 1 ? s.seg_c : s.stride_c;
    const float *in = s.nseg > 1 ? s.seg + ((size_t)seg * s.Be * s.heads + eh) * s.R * s.C : s.m_in ? s.m_in + eh * s.state : nullptr;
    float *out = STATE ? s.seg + ((size_t)seg * s.Be * s.heads + eh) * s.R * s.C : s.nseg > 1 || !s.m_out ? nullptr : s.m_out + eh * s.state;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < KS; i += 2) {
            const int r = w * KS + i, c = c0 + 32 * k + lane;
            const bool on = !STATE && in && c < s.C;
            M[k][i / 2] = pair_of(on && r < s.R ? in[r * sr + c * sc] : 0.f, on && r + 1 < s.R ? in[(r + 1) * sr + c * sc] : 0.f);
        }
    const int t_lo = seg * s.seg_len, t_hi = min(t_lo + s.seg_len, s.T);
    const int n0 = rev ? s.T - t_hi : t_lo, n1 = rev ? s.T - t_lo : t_hi;  // in the sweep's order
    int any = 0;
    // thread (j, l) fetches elements l, l + 32, ... of step j
    constexpr int RL = RP / 32, CL = kCols / 32;
    static_assert(kTokens == 8 && RP % 32 == 0, "a warp per step");
    const int j = w, l = lane;
    T fa[RL], fx[RL], fb[CL];
    int fg = 0;
    const auto fetch = [&](int n) {
        const bool on = n + j < n1;
        const long long row = on ? (long long)(rev ? s.T - 1 - (n + j) : n + j) * s.Be + e : 0;
#pragma unroll
        for (int i = 0; i < RL; ++i) {
            const int r = l + 32 * i;
            const bool ok = on && r < s.R;
            fa[i] = ok ? A[row * s.lda + r] : from_f32<T>(0.f);
            if (!STATE) fx[i] = ok ? X[row * s.ldx + r] : from_f32<T>(0.f);
        }
#pragma unroll
        for (int i = 0; i < CL; ++i) fb[i] = on && c0 + l + 32 * i < s.C ? B[row * s.ldb + l + 32 * i] : from_f32<T>(0.f);
        if (l == 0) fg = on && s.done && s.done[row] != 0;
    };
    fetch(n0);
    for (int n = n0; n < n1; n += kTokens) {
        const int cnt = min(kTokens, n1 - n);
        __syncthreads();  // the tile before is worked off
#pragma unroll
        for (int i = 0; i < RL; ++i)
        {
            ta[j][l + 32 * i] = to_f32(fa[i]) * s.a_scale;
            if (!STATE) tx[j][l + 32 * i] = to_f32(fx[i]);
        }
#pragma unroll
        for (int i = 0; i < CL; ++i) tb[j][l + 32 * i] = to_f32(fb[i]) * up[j];
        if (l == 0) gate[j] = fg;
        __syncthreads();
        if (n + kTokens < n1) fetch(n + kTokens);
        const auto steps = [&](auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            for (int t = 0; t < cnt; ++t) {
                const float b0 = tb[t][lane], b1 = tb[t][32 + lane];
                const pair32 b[2] = {pair_of(b0, b0), pair_of(b1, b1)};
                const int empty = gate[t];
                any |= empty;
                if (rev && empty) {
#pragma unroll
                    for (int i = 0; i < KS / 2; ++i) M[0][i] = M[1][i] = 0;
                }
                pair32 o[2] = {0, 0};
                const pair32 before = rev ? pair_of(1.f, 1.f) : pair_of(lam, lam);
#pragma unroll
                for (int i = 0; i < KS; i += 4) {
                    const ulonglong2 a = *reinterpret_cast<const ulonglong2 *>(&ta[t][w * KS + i]);
                    const ulonglong2 x = STATE ? make_ulonglong2(0, 0) : *reinterpret_cast<const ulonglong2 *>(&tx[t][w * KS + i]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        pair32 &m = M[q % 2][i / 2 + q / 2];
                        const pair32 aa = q < 2 ? a.x : a.y;
                        m = PLAIN ? fma2(before, m, mul2(aa, b[q % 2])) : fma2(aa, b[q % 2], m);
                        if constexpr (!STATE) o[q % 2] = fma2(q < 2 ? x.x : x.y, m, o[q % 2]);
                    }
                }
                if (rev ? PLAIN : empty) {
                    const pair32 after = pair_of(lam, lam);
#pragma unroll
                    for (int i = 0; i < KS / 2; ++i) {
                        M[0][i] = rev ? mul2(M[0][i], after) : 0;
                        M[1][i] = rev ? mul2(M[1][i], after) : 0;
                    }
                }
                if constexpr (!STATE) {
                    const float2 f0 = parts(o[0]), f1 = parts(o[1]);
                    part[w][t][lane] = f0.x + f0.y;
                    part[w][t][32 + lane] = f1.x + f1.y;
                }
            }
        };
        if (scaled) {
            const auto times = [&](float f) {
#pragma unroll
                for (int i = 0; i < KS / 2; ++i) {
                    M[0][i] = mul2(M[0][i], pair_of(f, f));
                    M[1][i] = mul2(M[1][i], pair_of(f, f));
                }
            };
            times(down[kTokens]);
            steps(std::false_type{});
            if (cnt < kTokens) times(exp2f((cnt - kTokens) * log2f(lam)));
        } else {
            steps(std::true_type{});
        }
        if constexpr (!STATE) {
            __syncthreads();
            for (int i = tid; i < cnt * kCols; i += 256) {
                const int t = i / kCols, c = i % kCols;
                if (c0 + c >= s.C) continue;
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < kSlices; ++k) v += part[k][t][c];
                v = v * down[t] * s.out_scale;
                const long long row = (long long)(rev ? s.T - 1 - (n + t) : n + t) * s.Be + e;
                if (s.shared) s.shared[(row * s.heads + h) * s.C + c0 + c] = v;
                else static_cast<T *>(s.out)[row * s.ldo + (long long)h * s.C + c0 + c] = from_f32<T>(v);
            }
        }
    }
    if (out) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < KS; i += 2) {
                const int r = w * KS + i, c = c0 + 32 * k + lane;
                const float2 f = parts(M[k][i / 2]);
                if (r < s.R && c < s.C) out[r * sr + c * sc] = f.x;
                if (r + 1 < s.R && c < s.C) out[(r + 1) * sr + c * sc] = f.y;
            }
    }
    if (STATE && c0 == 0 && tid == 0) s.seg_reset[(size_t)seg * s.Be * s.heads + eh] = any;
}
// KMOST: rows a warp of the sweep with the most, of 8 warps; fewer leave registers for more blocks on an SM.
template <typename T, bool STATE, int KMOST>
__global__ void __launch_bounds__(256, KMOST == 16 ? 2 : KMOST == 12 ? 3 : 4) sweep_kernel(const __grid_constant__ Sweeps all) {
    grid_wait();
    __shared__ __align__(16) StepTiles tile;
    const Sweep &s = all.s[blockIdx.z];
    if (blockIdx.x >= (s.C + kCols - 1) / kCols * s.Be * s.heads) return;
    if (s.R <= 32) sweep_rows<T, 4, STATE>(s, tile);
    else if (KMOST == 8 || s.R <= 64) sweep_rows<T, 8, STATE>(s, tile);
    else if (KMOST == 12 || s.R <= 96) sweep_rows<T, 12, STATE>(s, tile);
    else sweep_rows<T, 16, STATE>(s, tile);
}

// ---- one chunk of up to 64 steps on the tensor cores (bf16) ----
//
// Within a chunk of n steps, with i and j counted from its first one, w_ij = lambda^(i-j) and M the state in front of it,
//   out_i = sum_{j <= i} w_ij (x_i . a_j) b_j + lambda^(i+1) x_i^T M,    M <- lambda^n M + sum_j lambda^(n-1-j) a_j b_j^T
// (backwards one power less in the second and one more in the last term); terms with a reset between j and i, or between M and
// i, fall away.  Four products of 64-row tiles; the state stays in registers in 32 bits, 64 of its columns per block.
// Rounded to bf16: the weights w_ij (x_i . a_j), and the state where x reads it; half a step each, next to that of the output
// itself.  lambda^.. a_j is not: as one bf16 number it would leave 2^-8 in a state that is handed out in 32 bits; three terms hold
// the product in 32 bits, 2^-24 (in the kernel for many chunks two, 3 2^-16, where only outputs of bf16 come of it).
// A product has no masked places: 0 times a NaN of a later step would reach an earlier one, or stay behind a reset.  So a chunk that
// holds an infinity or a NaN is taken step by step, each as a chunk of its own, of which nothing is added where its flag is set.

constexpr int kChunk = 64, kBlockCols = 64;

__device__ __forceinline__ void mma_bf16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t *r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t *r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ float low(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float high(uint32_t p) { return __uint_as_float(p & 0xFFFF0000u); }
__device__ __forceinline__ bool not_finite(uint4 v) {  // one of eight bf16 numbers
    bool bad = false;
    for (uint32_t w : {v.x, v.y, v.z, v.w}) bad |= (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
    return bad;
}

// Shared memory: the tiles of X and A [64][RB + 8] and B [64][72] (rows padded by 16 bytes: ldmatrix without bank conflicts), M [RB][72],
// all bf16, then the powers of the decay.
template <int RB>
struct ChunkSmem {
    static constexpr int kRow = RB + 8, kCol = kBlockCols + 8;
    static constexpr int kWide = kChunk * kRow * 2, kNarrow = kChunk * kCol * 2, kState = RB * kCol * 2;
    static constexpr int kBytes = 2 * kWide + kNarrow + kState + 80 * 4;
};

// Sequences of 17 to 64 steps: one chunk.  RB: rows of the state, padded (64 or 128).
//
// Eight warps.  Outputs: warp (wr, wc) has 16 rows of the chunk and 32 columns; the two warps of the same rows both make their
// weights (a sixth more products than one alone, against an exchange).  State: warp w has 16 rows and all columns where there are
// 128 rows, else 16 rows and half of the columns.  Two blocks of 256 threads and 128 registers on an SM; with four warps and the
// whole state in theirs (240 registers) it is two of 128 threads, and an SM issues 1.3 to 1.7 instructions per cycle.
template <int RB>
__global__ void __launch_bounds__(256, 2) chunk_kernel(const __grid_constant__ Sweeps all) {
    grid_wait();
    const Sweep &s = all.s[blockIdx.z];
    using L = ChunkSmem<RB>;
    constexpr int TERMS = 3;
    constexpr int KR = RB / 16, MN = RB == 128 ? 8 : 4;  // 16-row steps of a product over R; column tiles of a warp's state
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t base = tc::smem_u32(smem);
    const uint32_t xs = base, as = xs + L::kWide, bs = as + L::kWide, ms_at = bs + L::kNarrow;
    uint8_t *ms = smem + 2 * L::kWide + L::kNarrow;
    float *pow = reinterpret_cast<float *>(ms + L::kState);
    const int tid = threadIdx.x, lane = tid % 32, w = tc::warp_index(), g = lane / 4, t4 = lane % 4;
    const int wr = w % 4, wc = w / 4, mr = RB == 128 ? 16 * w : 16 * wr, mc = RB == 128 ? 0 : 32 * wc;
    const int ncol = (s.C + kBlockCols - 1) / kBlockCols, c0 = blockIdx.x % ncol * kBlockCols, cols = min(kBlockCols, s.C - c0);
    const int eh = blockIdx.x / ncol, e = eh / s.heads, h = eh % s.heads, steps = s.T;
    if (e >= s.Be) return;  // another sweep of the launch has more columns
    const bf16 *A = static_cast<const bf16 *>(s.a) + (long long)(h / s.share_a) * s.R;
    const bf16 *B = static_cast<const bf16 *>(s.b) + (long long)(h / s.share_b) * s.C + c0;
    const bf16 *X = static_cast<const bf16 *>(s.x) + (long long)(h / s.share_x) * s.R;
    const int rev = s.reverse;
    if (tid < 66) pow[tid] = power(log2f(s.decay[h]), tid);

    // Rows first .. first + count of the sweep into rows 0 .., zeros behind them and behind R and C.
    auto copy = [&](int first, int count) {
        constexpr int WV = RB / 8, NV = kBlockCols / 8;
#pragma unroll
        for (int k = 0; k < kChunk * WV / 256; ++k) {
            const int i = k * 256 + tid, j = i / WV, v = i % WV, t = rev ? s.T - 1 - (first + j) : first + j;
            const bool ok = j < count && v * 8 < s.R;
            const long long row = ok ? (long long)t * s.Be + e : 0;
            tc::cp_async16(xs + (j * L::kRow + v * 8) * 2, ok ? X + row * s.ldx + v * 8 : X, ok);
            tc::cp_async16(as + (j * L::kRow + v * 8) * 2, ok ? A + row * s.lda + v * 8 : A, ok);
        }
#pragma unroll
        for (int k = 0; k < kChunk * NV / 256; ++k) {
            const int i = k * 256 + tid, j = i / NV, v = i % NV, t = rev ? s.T - 1 - (first + j) : first + j;
            const bool ok = j < count && v * 8 < cols;
            const long long row = ok ? (long long)t * s.Be + e : 0;
            tc::cp_async16(bs + (j * L::kCol + v * 8) * 2, ok ? B + row * s.ldb + v * 8 : B, ok);
        }
        tc::cp_async_commit();
    };
    copy(0, steps);

    // the state: rows mr + g (+ 8), columns mc + 8 n + 2 t4 (+ 1)
    const long long sr = s.stride_r, sc = s.stride_c;
    const float *in = s.m_in ? s.m_in + eh * s.state : nullptr;
    float *out_state = s.m_out ? s.m_out + eh * s.state : nullptr;
    float M[MN][4];
    auto at_state = [&](auto &&fn) {  // every place of the state that this thread holds, columns in pairs
#pragma unroll
        for (int n = 0; n < MN; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = mr + g + 8 * i, c = mc + 8 * n + 2 * t4;
                fn(M[n][2 * i], M[n][2 * i + 1], r < s.R && c < cols, r < s.R && c + 1 < cols, r * sr + (c0 + c) * sc);
            }
    };
    const bool pairs = sc == 1;  // pairs of columns are 8 aligned bytes: C is a multiple of 8
    at_state([&](float &m0, float &m1, bool ok0, bool ok1, long long at) {
        if (pairs) {
            const float2 f = in && ok0 ? *reinterpret_cast<const float2 *>(in + at) : make_float2(0.f, 0.f);
            m0 = f.x, m1 = f.y;
        } else {
            m0 = in && ok0 ? in[at] : 0.f;
            m1 = in && ok1 ? in[at + sc] : 0.f;
        }
    });
    bool filled = in != nullptr;  // M holds something

    // Whether what this thread has copied of B holds an infinity or a NaN.  (In X one reaches its own step's output, in A those it is
    // meant to; the weights that are masked, or zero, are set to zero whatever they come from.)
    auto odd = [&] {
        constexpr int NV = kBlockCols / 8;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kChunk * NV / 256; ++k) {
            const int i = k * 256 + tid;
            bad |= not_finite(*reinterpret_cast<const uint4 *>(smem + 2 * L::kWide + (i / NV * L::kCol + i % NV * 8) * 2));
        }
        return bad;
    };
    auto reset_at = [&](int step) { return s.done && step < steps && s.done[(long long)(rev ? s.T - 1 - step : step) * s.Be + e] != 0; };
    auto store_ms = [&] {  // M as an operand
#pragma unroll
        for (int n = 0; n < MN; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<uint32_t *>(ms + ((mr + g + 8 * i) * L::kCol + mc + 8 * n + 2 * t4) * 2) = pack_bf16x2(M[n][2 * i], M[n][2 * i + 1]);
    };

    // The n steps from `first` on, in rows 0 ..; resets: bit i set where done is at step first + i.
    auto process = [&](int first, int n, unsigned long long resets, bool last) {
        const auto before = [&](int i) { return __popcll(resets & (((1ull << i) << rev) - 1)); };  // resets in front of i
        if (16 * wr < n) {
            float o[4][4] = {};
            uint32_t xf[KR][4];
#pragma unroll
            for (int k = 0; k < KR; ++k) ldsm(xf[k], xs + ((16 * wr + lane % 16) * L::kRow + k * 16 + lane / 16 * 8) * 2);
            const int i0 = 16 * wr + g, i1 = i0 + 8;
            if (filled) {
#pragma unroll
                for (int k = 0; k < KR; ++k)
#pragma unroll
                    for (int nn = 0; nn < 2; ++nn) {
                        uint32_t b[4];
                        ldsm_t(b, ms_at + ((k * 16 + lane % 16) * L::kCol + wc * 32 + nn * 16 + lane / 16 * 8) * 2);
                        mma_bf16(o[2 * nn], xf[k], b[0], b[1]);
                        mma_bf16(o[2 * nn + 1], xf[k], b[2], b[3]);
                    }
                const bool on0 = resets == 0 || before(i0) == 0, on1 = resets == 0 || before(i1) == 0;
                const float f0 = pow[i0 + 1 - rev], f1 = pow[i1 + 1 - rev];
#pragma unroll
                for (int nn = 0; nn < 4; ++nn) {
                    o[nn][0] = on0 ? o[nn][0] * f0 : 0.f;
                    o[nn][1] = on0 ? o[nn][1] * f0 : 0.f;
                    o[nn][2] = on1 ? o[nn][2] * f1 : 0.f;
                    o[nn][3] = on1 ? o[nn][3] * f1 : 0.f;
                }
            }
            // 16 steps j at a time, up to the diagonal
#pragma unroll
            for (int js = 0; js < 4; ++js) {
                if (js > wr) break;
                float p[2][4] = {};
#pragma unroll
                for (int k = 0; k < KR; ++k) {
                    uint32_t b[4];
                    ldsm(b, as + ((js * 16 + lane / 16 * 8 + lane % 8) * L::kRow + k * 16 + lane / 8 % 2 * 8) * 2);
                    mma_bf16(p[0], xf[k], b[0], b[1]);
                    mma_bf16(p[1], xf[k], b[2], b[3]);
                }
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const int i = v < 2 ? i0 : i1, j = js * 16 + q * 8 + 2 * t4 + v % 2;
                        p[q][v] = i >= j ? p[q][v] * pow[max(i - j, 0)] : 0.f;
                    }
                if (resets != 0) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (before(v < 2 ? i0 : i1) != before(js * 16 + q * 8 + 2 * t4 + v % 2)) p[q][v] = 0.f;
                }
                const float f = s.a_scale;
                const uint32_t pf[4] = {pack_bf16x2(p[0][0] * f, p[0][1] * f), pack_bf16x2(p[0][2] * f, p[0][3] * f), pack_bf16x2(p[1][0] * f, p[1][1] * f),
                                        pack_bf16x2(p[1][2] * f, p[1][3] * f)};
#pragma unroll
                for (int nn = 0; nn < 2; ++nn) {
                    uint32_t b[4];
                    ldsm_t(b, bs + ((js * 16 + lane % 16) * L::kCol + wc * 32 + nn * 16 + lane / 16 * 8) * 2);
                    mma_bf16(o[2 * nn], pf, b[0], b[1]);
                    mma_bf16(o[2 * nn + 1], pf, b[2], b[3]);
                }
            }
            if (s.shared) {
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int i = v ? i1 : i0, t = rev ? s.T - 1 - (first + i) : first + i;
                    float *to = s.shared + (((long long)t * s.Be + e) * s.heads + h) * s.C + c0 + wc * 32;
                    if (i < n) {
#pragma unroll
                        for (int nn = 0; nn < 4; ++nn)
                            if (wc * 32 + 8 * nn + 2 * t4 < cols)
                                *reinterpret_cast<float2 *>(to + 8 * nn + 2 * t4) = make_float2(o[nn][2 * v] * s.out_scale, o[nn][2 * v + 1] * s.out_scale);
                    }
                }
            } else {
                // through the rows of X that only this warp and its neighbour read, to 64-byte rows of 16-byte stores
                uint8_t *mine = smem + (16 * wr * L::kRow + wc * 32) * 2;
                asm volatile("bar.sync %0, 64;" ::"r"(1 + wr) : "memory");  // both have read them
#pragma unroll
                for (int nn = 0; nn < 4; ++nn) {
                    *reinterpret_cast<uint32_t *>(mine + (g * L::kRow + 8 * nn + 2 * t4) * 2) = pack_bf16x2(o[nn][0] * s.out_scale, o[nn][1] * s.out_scale);
                    *reinterpret_cast<uint32_t *>(mine + ((g + 8) * L::kRow + 8 * nn + 2 * t4) * 2) = pack_bf16x2(o[nn][2] * s.out_scale, o[nn][3] * s.out_scale);
                }
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int r = k * 8 + lane / 4, v = lane % 4, i = 16 * wr + r, t = rev ? s.T - 1 - (first + i) : first + i;
                    if (i < n && wc * 32 + v * 8 < cols)
                        *reinterpret_cast<uint4 *>(static_cast<bf16 *>(s.out) + ((long long)t * s.Be + e) * s.ldo + (long long)h * s.C + c0 + wc * 32 + v * 8) =
                            *reinterpret_cast<const uint4 *>(mine + (r * L::kRow + v * 8) * 2);
                }
            }
        }
        if (last && !out_state) return;
        const float keep = pow[n];
        const int end = __popcll(resets);
#pragma unroll
        for (int nn = 0; nn < MN; ++nn)
#pragma unroll
            for (int v = 0; v < 4; ++v) M[nn][v] = resets == 0 ? M[nn][v] * keep : 0.f;
        if (n == 1 && resets != 0 && !rev) return;  // one step with its flag set: a product with weight 0 would let its NaN pass
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (16 * k >= n) break;
            uint32_t a[4], part[TERMS][4];
            ldsm_t(a, as + ((k * 16 + lane / 16 * 8 + lane % 8) * L::kRow + mr + lane / 8 % 2 * 8) * 2);
            float wj[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int j = 16 * k + 2 * t4 + v % 2 + v / 2 * 8;
                wj[v] = j < n && (resets == 0 || before(j) == end) ? pow[max(n - 1 - j + rev, 0)] * s.a_scale : 0.f;
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {  // a[v] holds steps 2 t4, 2 t4 + 1 (+ 8 in the upper two)
                float f0 = low(a[v]) * wj[v / 2 * 2], f1 = high(a[v]) * wj[v / 2 * 2 + 1];
                if (wj[v / 2 * 2] == 0.f) f0 = 0.f;
                if (wj[v / 2 * 2 + 1] == 0.f) f1 = 0.f;
#pragma unroll
                for (int q = 0; q < TERMS; ++q) {
                    part[q][v] = pack_bf16x2(f0, f1);
                    f0 -= low(part[q][v]);
                    f1 -= high(part[q][v]);
                }
            }
            // 16 steps are summed up by themselves and added to the state with a rounding to nearest: the tensor core cuts what it
            // adds to a larger number off, always downwards, which over thousands of steps shows
#pragma unroll
            for (int nn = 0; nn < MN / 2; ++nn) {
                uint32_t b[4];
                ldsm_t(b, bs + ((k * 16 + lane % 16) * L::kCol + mc + nn * 16 + lane / 16 * 8) * 2);
                float s0[4] = {}, s1[4] = {};
#pragma unroll
                for (int q = TERMS - 1; q >= 0; --q) {
                    mma_bf16(s0, part[q], b[0], b[1]);
                    mma_bf16(s1, part[q], b[2], b[3]);
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    M[2 * nn][v] += s0[v];
                    M[2 * nn + 1][v] += s1[v];
                }
            }
        }
    };

    const unsigned long long resets = (unsigned long long)__ballot_sync(0xffffffffu, reset_at(lane)) |
                                      (unsigned long long)__ballot_sync(0xffffffffu, reset_at(32 + lane)) << 32;
    if (filled) store_ms();
    tc::cp_async_wait<0>();
    const bool bad = __syncthreads_or(odd());
    for (int i = 0; i < (bad ? steps : 1); ++i) {
        if (bad) {
            __syncthreads();
            copy(i, 1);
            tc::cp_async_wait<0>();
            if (filled) store_ms();
            __syncthreads();
        }
        process(i, bad ? 1 : steps, bad ? resets >> i & 1 : resets, !bad || i == steps - 1);
        filled = true;
    }
    if (!out_state) return;
    at_state([&](float &m0, float &m1, bool ok0, bool ok1, long long at) {
        if (pairs) {
            if (ok0) *reinterpret_cast<float2 *>(out_state + at) = make_float2(m0, m1);
        } else {
            if (ok0) out_state[at] = m0;
            if (ok1) out_state[at + sc] = m1;
        }
    });
}

// Sequences of up to 16 steps: one chunk, four warps, and little else than the state to move, so as many blocks on an SM as keep its
// loads in flight.  Every warp makes the 16 x 16 weights and has 16 columns of the outputs; of the state it has RB / 4 rows.  16 steps
// of 256 x 16 heads of 64 x 64: 50 us, 3.3 TB/s (by chunk_kernel 71): six blocks of an SM wait for their first loads and store at their end.
template <int RB>
__global__ void __launch_bounds__(128, RB == 64 ? 6 : 3) short_kernel(const __grid_constant__ Sweeps all) {
    grid_wait();
    const Sweep &s = all.s[blockIdx.z];
    constexpr int TERMS = 3;
    constexpr int kRow = RB + 8, kCol = kBlockCols + 8, KR = RB / 16, MT = RB / 64;
    __shared__ __align__(16) bf16 xs[16 * kRow], as[16 * kRow], bs[16 * kCol], ms[RB * kCol];
    __shared__ float pow[20];
    const int tid = threadIdx.x, lane = tid % 32, w = tc::warp_index(), g = lane / 4, t4 = lane % 4;
    const int ncol = (s.C + kBlockCols - 1) / kBlockCols, c0 = blockIdx.x % ncol * kBlockCols, cols = min(kBlockCols, s.C - c0);
    const int eh = blockIdx.x / ncol, e = eh / s.heads, h = eh % s.heads, rev = s.reverse, n = s.T;
    if (e >= s.Be) return;  // another sweep of the launch has more columns
    const bf16 *A = static_cast<const bf16 *>(s.a) + (long long)(h / s.share_a) * s.R;
    const bf16 *B = static_cast<const bf16 *>(s.b) + (long long)(h / s.share_b) * s.C + c0;
    const bf16 *X = static_cast<const bf16 *>(s.x) + (long long)(h / s.share_x) * s.R;

    // rows 64 m + 16 w + g (+ 8), columns 8 n + 2 t4 (+ 1)
    const bool pairs = s.stride_c == 1;
    float M[MT][8][4];
    auto at_state = [&](auto &&fn) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = 64 * m + 16 * w + g + 8 * i, c = 8 * k + 2 * t4;
                    fn(M[m][k][2 * i], M[m][k][2 * i + 1], r < s.R && c < cols, r * s.stride_r + (c0 + c) * s.stride_c);
                }
    };
    const float *in = s.m_in ? s.m_in + eh * s.state : nullptr;
    if (in)
        at_state([&](float &m0, float &m1, bool ok, long long at) {
            if (pairs) {
                const float2 f = ok ? __ldcs(reinterpret_cast<const float2 *>(in + at)) : make_float2(0.f, 0.f);
                m0 = f.x, m1 = f.y;
            } else {
                m0 = ok ? __ldcs(in + at) : 0.f;
                m1 = ok ? __ldcs(in + at + s.stride_c) : 0.f;
            }
        });
    else at_state([&](float &m0, float &m1, bool, long long) { m0 = m1 = 0.f; });

    auto copy = [&](int first, int count) {  // as in chunk_kernel
        constexpr int WV = RB / 8, NV = kBlockCols / 8;
        for (int i = tid; i < 16 * WV; i += 128) {
            const int j = i / WV, v = i % WV, t = rev ? s.T - 1 - (first + j) : first + j;
            const bool ok = j < count && v * 8 < s.R;
            const long long row = ok ? (long long)t * s.Be + e : 0;
            tc::cp_async16(tc::smem_u32(xs + j * kRow + v * 8), ok ? X + row * s.ldx + v * 8 : X, ok);
            tc::cp_async16(tc::smem_u32(as + j * kRow + v * 8), ok ? A + row * s.lda + v * 8 : A, ok);
        }
        {
            const int j = tid / NV, v = tid % NV, t = rev ? s.T - 1 - (first + j) : first + j;
            const bool ok = j < count && v * 8 < cols;
            const long long row = ok ? (long long)t * s.Be + e : 0;
            tc::cp_async16(tc::smem_u32(bs + j * kCol + v * 8), ok ? B + row * s.ldb + v * 8 : B, ok);
        }
        tc::cp_async_commit();
        tc::cp_async_wait<0>();
    };
    copy(0, n);
    const bool flag = s.done && lane < n && s.done[(long long)(rev ? s.T - 1 - lane : lane) * s.Be + e] != 0;
    const uint32_t resets_all = __ballot_sync(0xffffffffu, flag);
    if (tid < 18) pow[tid] = power(log2f(s.decay[h]), tid);
    const bool bad = __syncthreads_or(not_finite(*reinterpret_cast<const uint4 *>(bs + tid / 8 * kCol + tid % 8 * 8)));
    bool filled = in != nullptr;
    for (int piece = 0; piece < (bad ? n : 1); ++piece) {
        const int count = bad ? 1 : n, first = bad ? piece : 0;
        const uint32_t resets = bad ? resets_all >> piece & 1 : resets_all;
        if (bad) {
            __syncthreads();
            copy(piece, 1);
        }
        if (filled) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        *reinterpret_cast<uint32_t *>(ms + (64 * m + 16 * w + g + 8 * i) * kCol + 8 * k + 2 * t4) = pack_bf16x2(M[m][k][2 * i], M[m][k][2 * i + 1]);
        }
        __syncthreads();
        const auto before = [&](int i) { return __popc(resets & (((1u << i) << rev) - 1)); };
        {
            float o[2][4] = {}, p[2][4] = {};
#pragma unroll
            for (int k = 0; k < KR; ++k) {
                uint32_t xf[4], b[4];
                ldsm(xf, tc::smem_u32(xs + (lane % 16) * kRow + k * 16 + lane / 16 * 8));
                ldsm(b, tc::smem_u32(as + (lane / 16 * 8 + lane % 8) * kRow + k * 16 + lane / 8 % 2 * 8));
                mma_bf16(p[0], xf, b[0], b[1]);
                mma_bf16(p[1], xf, b[2], b[3]);
                if (filled) {
                    ldsm_t(b, tc::smem_u32(ms + (k * 16 + lane % 16) * kCol + 16 * w + lane / 16 * 8));
                    mma_bf16(o[0], xf, b[0], b[1]);
                    mma_bf16(o[1], xf, b[2], b[3]);
                }
            }
            const bool on0 = before(g) == 0, on1 = before(g + 8) == 0;
            const float f0 = pow[g + 1 - rev], f1 = pow[g + 9 - rev];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                o[q][0] = on0 ? o[q][0] * f0 : 0.f;
                o[q][1] = on0 ? o[q][1] * f0 : 0.f;
                o[q][2] = on1 ? o[q][2] * f1 : 0.f;
                o[q][3] = on1 ? o[q][3] * f1 : 0.f;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int i = v < 2 ? g : g + 8, j = q * 8 + 2 * t4 + v % 2;
                    p[q][v] = i >= j && before(i) == before(j) ? p[q][v] * (pow[max(i - j, 0)] * s.a_scale) : 0.f;
                }
            }
            const uint32_t pf[4] = {pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]), pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3])};
            uint32_t b[4];
            ldsm_t(b, tc::smem_u32(bs + (lane % 16) * kCol + 16 * w + lane / 16 * 8));
            mma_bf16(o[0], pf, b[0], b[1]);
            mma_bf16(o[1], pf, b[2], b[3]);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int i = g + 8 * v, t = rev ? s.T - 1 - (first + i) : first + i;
                const long long row = (long long)t * s.Be + e;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int c = 16 * w + 8 * q + 2 * t4;
                    if (i >= count || c >= cols) continue;
                    const float o0 = o[q][2 * v] * s.out_scale, o1 = o[q][2 * v + 1] * s.out_scale;
                    if (s.shared) *reinterpret_cast<float2 *>(s.shared + (row * s.heads + h) * s.C + c0 + c) = make_float2(o0, o1);
                    else *reinterpret_cast<uint32_t *>(static_cast<bf16 *>(s.out) + row * s.ldo + (long long)h * s.C + c0 + c) = pack_bf16x2(o0, o1);
                }
            }
        }
        filled = true;
        if (!s.m_out && (!bad || piece == n - 1)) continue;
        const int end = __popc(resets);
        const float keep = pow[count];
        if (count == 1 && resets != 0 && !rev) {  // nothing of the step is left; a product with weight 0 would let its NaN pass
            __syncthreads();
            if (tid < kBlockCols) bs[tid] = from_f32<bf16>(0.f);
            __syncthreads();
        }
        float wj[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int j = 2 * t4 + v % 2 + v / 2 * 8;
            wj[v] = j < count && before(j) == end ? pow[max(count - 1 - j + rev, 0)] * s.a_scale : 0.f;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            uint32_t a[4], part[TERMS][4];
            ldsm_t(a, tc::smem_u32(as + (lane / 16 * 8 + lane % 8) * kRow + 64 * m + 16 * w + lane / 8 % 2 * 8));
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float f0 = low(a[v]) * wj[v / 2 * 2], f1 = high(a[v]) * wj[v / 2 * 2 + 1];
                if (wj[v / 2 * 2] == 0.f) f0 = 0.f;
                if (wj[v / 2 * 2 + 1] == 0.f) f1 = 0.f;
#pragma unroll
                for (int q = 0; q < TERMS; ++q) {
                    part[q][v] = pack_bf16x2(f0, f1);
                    f0 -= low(part[q][v]);
                    f1 -= high(part[q][v]);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t b[4];
                ldsm_t(b, tc::smem_u32(bs + (lane % 16) * kCol + k * 16 + lane / 16 * 8));
                float s0[4] = {}, s1[4] = {};
#pragma unroll
                for (int q = TERMS - 1; q >= 0; --q) {
                    mma_bf16(s0, part[q], b[0], b[1]);
                    mma_bf16(s1, part[q], b[2], b[3]);
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    M[m][2 * k][v] = resets == 0 ? fmaf(M[m][2 * k][v], keep, s0[v]) : s0[v];
                    M[m][2 * k + 1][v] = resets == 0 ? fmaf(M[m][2 * k + 1][v], keep, s1[v]) : s1[v];
                }
            }
        }
    }
    if (!s.m_out) return;
    float *out = s.m_out + eh * s.state;
    at_state([&](float &m0, float &m1, bool ok, long long at) {
        if (!ok) return;
        if (pairs) {
            __stcs(reinterpret_cast<float2 *>(out + at), make_float2(m0, m1));
        } else {
            __stcs(out + at, m0);
            __stcs(out + at + s.stride_c, m1);
        }
    });
}

// ---- chunks of 128 steps on tcgen05 (bf16, more than 64 steps) ----
//
// The same four products as tcgen05.mma with accumulators in tensor memory, whole heads per block: S = X A^T and O1 = X M as soon as the
// rows have landed; K = (w A)^T B while S is weighted into P; O2 = P B.  One warp moves tiles (TMA) and issues the products; the
// others are between them: a thread owns a row of each accumulator (a step, or a row of the state) and a part of its columns.  Operands lie
// in panels of 64 columns, 128 bytes a row, swizzled: A is read along its rows for S and down its columns (MN-major) for K.  The state
// stays in registers in 32 bits; M is its bf16 image.  Rows of a tile are steps in time's order; backwards, the chunks and the masks turn
// round.
//   64 rows: the weighted keys' first two terms are the two halves of a 128-row operand, and what comes of them stays apart, as rows r
// and 64 + r of the state, which X reads one after the other: their sum is made once, at the end.
// mma.sync at these sizes is bound by what goes with it, 13 instructions for each product (8192 steps of 16 x 128: 219 us, here 85).
// Bound by the steps of a chunk one after another (tiles, S, P, O2, outputs) with one or two blocks on an SM to cover them: 6 to 8 thousand
// cycles of a chunk, of which the products are one and all traffic of shared memory three; blocks of 64 x 64 run two to an SM.  Only O1
// needs the state in front of the chunk: S, the split and K could be made a chunk ahead, and are not.

// RB, CB: rows and columns of the state, padded to 64 or 128.  STATE: only what the segment leaves, from an empty state.  TERMS: of the
// weighted a.
template <int RB, int CB, bool STATE, int TERMS>
struct TileSmem {
    static constexpr int kPanel = 128 * 128;  // bytes: 128 rows of 64 bf16 numbers
    // P takes the place of X, and where that is one panel, of A behind it.  With 128 rows there is room for X of the next chunk
    // (with three terms there is not), and A's place is free once it is split.  With 64 X and A change places with the first two terms
    // from chunk to chunk: these are free once K is made, long before the outputs have left P's place (gradients 2048 x 4 x 16 x 64: 154 -> 137 us, with
    // 16 columns of the accumulators at a time).
    static constexpr bool kAhead = RB == 128 && TERMS == 2 && !STATE, kTurns = RB == 64 && !STATE;
    __device__ static int x_at(int i) { return kAhead ? kX + i % 2 * kWide : kTurns && i % 2 ? kSplit : kX; }
    __device__ static int a_at(int i) { return kTurns ? x_at(i) + kPanel : kA; }
    __device__ static int split_at(int i, int panel) { return kTurns && i % 2 && panel < 2 ? kX + panel * kPanel : kSplit + panel * kPanel; }
    static constexpr int kWide = RB / 64 * kPanel, kX = 0, kA = kX + (STATE ? 0 : (kAhead ? 2 : 1) * kWide), kB = kA + kWide, kM = kB + CB / 64 * kPanel,
                         kSplit = kM + (STATE ? 0 : CB / 64 * kPanel), kSplitBytes = RB == 128 ? TERMS * 2 * kPanel : TERMS * kPanel,
                         kEnd = kSplit + kSplitBytes;
    static constexpr int kTables = 1680, kBytes = kEnd + kTables + 1024;  // with the alignment
    static constexpr uint32_t kCols = STATE ? CB : 128 + 2 * CB > 256 ? 512 : 256;  // of tensor memory
    static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};
struct TileTables {
    float weight[256];  // a_scale lambda^|p - c| of step c for step p at 127 - p + c
    float pow[132];     // lambda^n
    uint64_t got_a, got_b, bar[3];    // X and A, B have landed; S and O1, K, O2 are made
    // of the workers' warps: A is split; B is looked at, and with outputs P is there; accumulators are read, M and outputs in place
    uint64_t split, weighted, emptied;
    uint64_t left;                      // outputs have left shared memory (kTurns)
    uint32_t flags[2][4];  // done at the steps of a chunk, a bit each
    int abort_flag, bad;
    uint32_t slot;
};
static_assert(sizeof(TileTables) <= 1680, "place of the tables");

// w a for eight bf16 numbers a, as sums of bf16 numbers.  With w = w0 + w1 + w2, 8 bits each, hi = a w0 to the nearest and a w0 - hi are
// bf16 numbers that hold a w0 entirely (16 bits), in two packed operations a pair; four terms are off by less than 2^-23 (at most
// 0.72 2^-24 of 2 million), two by less than 3 2^-16 (1.64).  Three come from 32 bits, 17 operations a pair, and are off by 2^-24: with 128
// rows, where the fourth would cost more products and shared memory than it saves (8192 steps of 16 x 128: 97 and 90 us).
template <int TERMS>
__device__ __forceinline__ void split_products(const uint32_t (&a)[4], float w, uint32_t (&part)[TERMS][4]) {
    if constexpr (TERMS == 3) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f0 = low(a[q]) * w, f1 = high(a[q]) * w;
#pragma unroll
            for (int t = 0; t < 3; ++t) {
                part[t][q] = pack_bf16x2(f0, f1);
                f0 -= low(part[t][q]);
                f1 -= high(part[t][q]);
            }
        }
    } else {
        __nv_bfloat162 ws[3];
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            ws[t] = __float2bfloat162_rn(w);
            w -= __low2float(ws[t]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&a[q]);
            __nv_bfloat162 p[4];
            p[0] = __hmul2_rn(x, ws[0]);
            p[1] = __hfma2(x, ws[0], __hneg2(p[0]));
            if constexpr (TERMS == 2) {
                p[1] = __hfma2(x, ws[1], p[1]);
            } else {
                p[2] = __hmul2_rn(x, ws[1]);
                p[3] = __hfma2(x, ws[2], __hfma2(x, ws[1], __hneg2(p[2])));
            }
#pragma unroll
            for (int t = 0; t < TERMS; ++t) part[t][q] = *reinterpret_cast<const uint32_t *>(&p[t]);
        }
    }
}
__device__ __forceinline__ void store_32_bytes(float *p, const float *v) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]),
                 "f"(v[6]), "f"(v[7])
                 : "memory");
}

struct TileMap {
    CUtensorMap x, a, b, out;
};
struct TileMaps {
    TileMap m[3];
};

// The segment step by step, a thread per column: what infinities and NaN in B are left to, which a product of masked weights would let
// reach steps that do not see them.
template <bool STATE>
__device__ __noinline__ void segment_slowly(const Sweep &s, float *m, const float *in, float *out_state, long long sr, long long sc, int eh, int t_lo,
                                            int t_hi) {
    const int e = eh / s.heads, h = eh % s.heads, c = threadIdx.x, rev = s.reverse;
    const float lam = s.decay[h];
    if (c >= s.C) return;
    for (int r = 0; r < s.R; ++r) m[r * s.C + c] = in ? in[r * sr + c * sc] : 0.f;
    for (int n = 0; n < t_hi - t_lo; ++n) {
        const int t = rev ? t_hi - 1 - n : t_lo + n;
        const long long row = (long long)t * s.Be + e;
        const bool gate = s.done && s.done[row] != 0;
        const bf16 *a = static_cast<const bf16 *>(s.a) + row * s.lda + (long long)(h / s.share_a) * s.R;
        const bf16 *x = static_cast<const bf16 *>(s.x) + row * s.ldx + (long long)(h / s.share_x) * s.R;
        const float b = bf2f(static_cast<const bf16 *>(s.b)[row * s.ldb + (long long)(h / s.share_b) * s.C + c]);
        float o = 0.f;
        for (int r = 0; r < s.R; ++r) {
            float v = m[r * s.C + c];
            v = rev ? (gate ? 0.f : v) : v * lam;
            v = fmaf(bf2f(a[r]) * s.a_scale, b, v);
            if (!STATE) o = fmaf(bf2f(x[r]), v, o);
            m[r * s.C + c] = rev ? v * lam : gate ? 0.f : v;
        }
        if (STATE) continue;
        o *= s.out_scale;
        if (s.shared) s.shared[(row * s.heads + h) * s.C + c] = o;
        else static_cast<bf16 *>(s.out)[row * s.ldo + (long long)h * s.C + c] = __float2bfloat16_rn(o);
    }
    if (out_state)
        for (int r = 0; r < s.R; ++r) out_state[r * sr + c * sc] = m[r * s.C + c];
}

// A warp for tiles and products, and workers: eight warps of two blocks on an SM, or sixteen of one (eight where there are no outputs:
// 128 x 128, eight and sixteen: 36 and 40 us of states, 54 and 48 of outputs).
__host__ __device__ constexpr int tile_threads(int RB, int CB, bool STATE) { return STATE || (RB == 64 && CB == 64) ? 288 : 544; }
template <int N>
__device__ __forceinline__ void tmem_get(uint32_t at, float *v) {
    if constexpr (N == 16) tc::tmem_ld16(at, v);
    else tc::tmem_ld32(at, v);
}

template <int RB, int CB, bool STATE, int TERMS>
__global__ void __launch_bounds__(tile_threads(RB, CB, STATE), RB == 64 && CB == 64 ? 2 : 1) tile_kernel(const __grid_constant__ Sweeps all, const __grid_constant__ TileMaps all_maps,
                                                                                int32_t *status) {
    const Sweep &s = all.s[blockIdx.z];
    const TileMap &maps = all_maps.m[blockIdx.z];
    using L = TileSmem<RB, CB, STATE, TERMS>;
    constexpr int WG = (tile_threads(RB, CB, STATE) - 32) / 128, WORKERS = 128 * WG;  // warps 0 ..; column groups
    constexpr int H = CB / WG, PC = 128 / WG;            // columns of a thread: of the state and the outputs, of S and P
    constexpr int G = STATE && H >= 32 ? 32 : 16;        // at a time: with outputs there are registers for 16 of two accumulators
    constexpr int kO1 = 128, kK = STATE ? 0 : 128 + CB;  // columns of tensor memory: S and O2 from 0
    constexpr int SETS = RB == 128 ? TERMS : TERMS / 2;
    static_assert(RB == 128 || TERMS != 3, "two terms side by side");
    extern __shared__ uint8_t raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    TileTables *tab = reinterpret_cast<TileTables *>(smem + L::kEnd);
    const uint32_t base = tc::smem_u32(smem);
    const int tid = threadIdx.x, lane = tid % 32, w = tc::warp_index();
    volatile int *abort_flag = &tab->abort_flag;
    if (w == 4 * WG) {  // the warp that uses them first
        if (lane == 0) {
            tc::mbar_init(&tab->got_a, 1);
            tc::mbar_init(&tab->got_b, 1);
            for (int i = 0; i < 3; ++i) tc::mbar_init(&tab->bar[i], 1);
            tc::mbar_init(&tab->split, 4 * WG);
            tc::mbar_init(&tab->weighted, 4 * WG);
            tc::mbar_init(&tab->emptied, 4 * WG);
            tc::mbar_init(&tab->left, 1);
            tab->abort_flag = tab->bad = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }
    if (w == 4 * WG) tc::tmem_alloc(&tab->slot, L::kCols);
    grid_wait();
    const int eh = blockIdx.x, e = eh / s.heads, h = eh % s.heads, seg = blockIdx.y, rev = s.reverse;
    const int t_lo = seg * s.seg_len, t_hi = min(t_lo + s.seg_len, s.T), chunks = (t_hi - t_lo + 127) / 128;
    if (tid < 256) {
        const float l2 = log2f(s.decay[h]);
        const int d = rev ? tid - 127 : 127 - tid;  // steps between
        tab->weight[tid] = d < 0 ? 0.f : power(l2, d) * s.a_scale;
        if (tid < 130) tab->pow[tid] = power(l2, tid);
    }
    const long long sr = s.nseg > 1 ? s.seg_r : s.stride_r, sc = s.nseg > 1 ? s.seg_c : s.stride_c;
    const long long place = s.nseg > 1 ? ((long long)seg * s.Be * s.heads + eh) * s.R * s.C : eh * s.state;
    const float *in = STATE ? nullptr : s.nseg > 1 ? s.seg + place : s.m_in ? s.m_in + place : nullptr;
    float *out_state = STATE ? s.seg + place : s.nseg > 1 || !s.m_out ? nullptr : s.m_out + place;
    const auto start_of = [&](int i) { return t_lo + 128 * (rev ? chunks - 1 - i : i); };  // of the i-th chunk
    bool ok = true;

    if (w == 4 * WG) {
        // ---------------- tiles and products
        const auto load = [&](int to, const CUtensorMap *map, int width, int head, int t, uint64_t *bar) {
            for (int p = 0; p < width / 64; ++p) tc::tma_load_4d(base + to + p * L::kPanel, map, bar, 64 * p, head, e, t);
        };
        const auto load_x = [&](int i) { load(L::x_at(i), &maps.x, RB, h / s.share_x, start_of(i), &tab->got_a); };
        const auto load_a = [&](int i) { load(L::a_at(i), &maps.a, RB, h / s.share_a, start_of(i), &tab->got_a); };
        const auto load_b = [&](int i) { load(L::kB, &maps.b, CB, h / s.share_b, start_of(i), &tab->got_b); };
        // done at the steps of the i-th chunk, for the workers; in front of the arrival that they wait for
        const auto flags_of = [&](int i) {
            const int t0 = start_of(i);
            uint8_t f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = t0 + 32 * k + lane;
                f[k] = s.done && t < t_hi ? s.done[(long long)t * s.Be + e] : 0;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t word = __ballot_sync(0xffffffffu, f[k] != 0);
                if (lane == 0) tab->flags[i % 2][k] = word;
            }
            __syncwarp();
        };
        const auto expect_a = [&] { tc::mbar_arrive_expect_tx(&tab->got_a, (STATE ? 1 : 2) * L::kWide); };
        const auto expect_b = [&] { tc::mbar_arrive_expect_tx(&tab->got_b, CB / 64 * L::kPanel); };
        flags_of(0);
        if (tc::elect_one()) {
            expect_a();
            if (!STATE) load_x(0);
            load_a(0);
            expect_b();
            load_b(0);
        }
        __syncwarp();
        tc::tc_fence_before();
        __syncthreads();
        tc::tc_fence_after();
        const uint32_t tmem = tab->slot;
        // Descriptors: along the rows (K-major), and down the columns (MN-major, panels side by side).
        const uint64_t dk = tc::smem_desc_sw(base, 16, 1024, 128), dm = tc::smem_desc_sw(base, L::kPanel, 1024, 128);
        const uint32_t k_hi = (uint32_t)(dk >> 32), m_hi = (uint32_t)(dm >> 32), k_lo = (uint32_t)dk, m_lo = (uint32_t)dm;
        const auto along = [&](int panel, int k) { return k_lo + (uint32_t)(panel >> 4) + 2u * k; };     // step k of 16 columns of one panel
        const auto down = [&](int panels, int k) { return m_lo + (uint32_t)(panels >> 4) + 128u * k; };  // step k of 16 rows
        const auto wait = [&](uint64_t *bar, int i) { ok = tc::mbar_wait_warp(bar, i & 1, abort_flag, status) && ok; };
        bool filled = in != nullptr;
        for (int i = 0; i < chunks; ++i) {
            const bool more = i + 1 < chunks, update = more || out_state;
            const int x = L::x_at(i), at_a = L::a_at(i);
            if (!STATE) {
                wait(&tab->got_a, i);
                tc::tc_fence_after();
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < RB / 16; ++k)
                        tc::umma_bf16_lh(tmem, along(x + k / 4 * L::kPanel, k % 4), k_hi, along(at_a + k / 4 * L::kPanel, k % 4), k_hi,
                                         tc::instr_desc(128, 128, 0, 0), k > 0);
                    if (filled) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int xk = k % (RB / 16);
                            tc::umma_bf16_lh(tmem + kO1, along(x + xk / 4 * L::kPanel, xk % 4), k_hi, down(L::kM, k), m_hi, tc::instr_desc(128, CB, 0, 1), k > 0);
                        }
                    }
                    tc::umma_commit(&tab->bar[0]);
                }
                __syncwarp();
            }
            if (more) flags_of(i + 1);
            if (L::kAhead && more && tc::elect_one()) {
                tc::bulk_wait_read<0>();  // the chunk before has left that place
                expect_a();
                load_x(i + 1);
            }
            __syncwarp();
            wait(&tab->split, i);
            if (update) {
                wait(&tab->got_b, i);
                tc::tc_fence_after();
                if (tc::elect_one()) {
#pragma unroll
                    for (int t = SETS - 1; t >= 0; --t)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            tc::umma_bf16_lh(tmem + kK, down(L::split_at(i, 2 * t), k), m_hi, down(L::kB, k), m_hi, tc::instr_desc(128, CB, 1, 1),
                                             t < SETS - 1 || k > 0);
                    tc::umma_commit(&tab->bar[1]);
                }
                __syncwarp();
                if (L::kTurns && more) {
                    wait(&tab->bar[1], i);  // K is made
                    if (tc::elect_one()) {
                        expect_a();
                        load_x(i + 1);
                        load_a(i + 1);
                    }
                    __syncwarp();
                }
            }
            if (STATE && more && tc::elect_one()) {
                expect_a();
                load_a(i + 1);
            }
            __syncwarp();
            if (!STATE) {
                if (L::kAhead && more) {
                    wait(&tab->bar[0], i);  // S is made
                    if (tc::elect_one()) load_a(i + 1);
                    __syncwarp();
                }
                wait(&tab->weighted, i);
                if (!update) wait(&tab->got_b, i);
                tc::tc_fence_after();
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        tc::umma_bf16_lh(tmem, along(x + k / 4 * L::kPanel, k % 4), k_hi, down(L::kB, k), m_hi, tc::instr_desc(128, CB, 0, 1), k > 0);
                    tc::umma_commit(&tab->bar[2]);
                }
                __syncwarp();
            }
            if (more) {  // all that reads B is made, and the workers have looked at it
                wait(&tab->bar[STATE ? 1 : 2], i);
                if (STATE) wait(&tab->weighted, i);
                if (tc::elect_one()) {
                    expect_b();
                    load_b(i + 1);
                }
                __syncwarp();
            }
            wait(&tab->emptied, i);
            tc::tc_fence_after();
            if (!STATE && tc::elect_one()) {
                if (!s.shared) {
                    for (int p = 0; p < CB / 64; ++p)
                        if (64 * p < s.C) tc::tma_store_4d(&maps.out, base + x + p * L::kPanel, 64 * p, h, e, start_of(i));
                    tc::bulk_commit();
                }
                if (L::kTurns) {
                    tc::bulk_wait_read<0>();
                    tc::mbar_arrive(&tab->left);
                } else if (!L::kAhead && more) {
                    tc::bulk_wait_read<0>();
                    expect_a();
                    load_x(i + 1);
                    load_a(i + 1);
                }
            }
            __syncwarp();
            filled = true;
        }
        if (!STATE && tc::elect_one()) tc::bulk_wait_all();
        __syncwarp();
        if (!ok) {  // copies in flight land meanwhile
            const long long t0 = clock64();
            while (clock64() - t0 < 200000) {
            }
        }
    } else {
        // ---------------- what is between the products
        const int lq = w % 4, wc = w / 4, row = 32 * lq + lane;
        // row `row` of the state (with 64: rows 64 .. are the second terms' share), columns wc H ..
        float M[H];
        const bool mine_on = row < s.R && (RB == 128 || row < 64);
        {
            const bool on = in && mine_on;
            const float *p = in + row * sr + wc * H * sc;
            if (sc == 1) {
#pragma unroll
                for (int c = 0; c < H; c += 4) {
                    const float4 f = on && wc * H + c < s.C ? *reinterpret_cast<const float4 *>(p + c) : make_float4(0.f, 0.f, 0.f, 0.f);
                    M[c] = f.x, M[c + 1] = f.y, M[c + 2] = f.z, M[c + 3] = f.w;
                }
            } else {
#pragma unroll
                for (int c = 0; c < H; ++c) M[c] = on && wc * H + c < s.C ? p[c * sc] : 0.f;
            }
        }
        const auto piece = [&](int panel, int r, int v) { return smem + panel + r * 128 + ((v ^ r) & 7) * 16; };
        const auto store_m = [&] {
#pragma unroll
            for (int c = 0; c < H; c += 8) {
                const int v = (wc * H + c) / 8;
                *reinterpret_cast<uint4 *>(piece(L::kM + v / 8 * L::kPanel, row, v)) =
                    make_uint4(pack_bf16x2(M[c], M[c + 1]), pack_bf16x2(M[c + 2], M[c + 3]), pack_bf16x2(M[c + 4], M[c + 5]), pack_bf16x2(M[c + 6], M[c + 7]));
            }
        };
        bool filled = in != nullptr;
        __nv_bfloat162 zeros = __float2bfloat162_rn(0.f);  // of all of B that this thread looks at
        if (!STATE && filled) store_m();
        tc::fence_async_smem();
        tc::tc_fence_before();
        __syncthreads();
        tc::tc_fence_after();
        const uint32_t mine = tab->slot + ((uint32_t)(32 * lq) << 16);
        const auto wait = [&](uint64_t *bar, int i) { ok = tc::mbar_wait(bar, i & 1, abort_flag, status) && ok; };
        const auto tell = [&](uint64_t *bar) {
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bar);
        };
        uint32_t any = 0;
        for (int i = 0; i < chunks; ++i) {
            const int n = min(128, t_hi - start_of(i));
            const bool more = i + 1 < chunks, update = more || out_state;
            const int x = L::x_at(i), at_a = L::a_at(i);
            wait(&tab->got_a, i);
            uint32_t resets[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) any |= resets[k] = tab->flags[i % 2][k];
            const bool some = (resets[0] | resets[1] | resets[2] | resets[3]) != 0;
            // the flag that the state behind the chunk sees first, looking back
            int edge = rev ? 128 : -1;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!rev && resets[k]) edge = 32 * k + 31 - __clz(resets[k]);
                if (rev && resets[3 - k]) edge = 32 * (3 - k) + __ffs(resets[3 - k]) - 1;
            }
            if (L::kTurns && i > 0) wait(&tab->left, i - 1);  // the split terms' place
            if (update) {
                // w_c a_c in TERMS terms
                constexpr int V = RB / 8;
#pragma unroll 4
                for (int k = 0; k < 128 * V / WORKERS; ++k) {
                    const int c = (k * WORKERS + tid) / V, v = (k * WORKERS + tid) % V;
                    const bool sees = c < n && (rev ? c <= edge : c > edge);
                    const float wj = sees ? tab->pow[max(rev ? c + 1 : n - 1 - c, 0)] * s.a_scale : 0.f;
                    const uint4 a = *reinterpret_cast<const uint4 *>(piece(at_a + v / 8 * L::kPanel, c, v));
                    const uint32_t in4[4] = {sees ? a.x : 0u, sees ? a.y : 0u, sees ? a.z : 0u, sees ? a.w : 0u};
                    uint32_t part[TERMS][4];
                    split_products<TERMS>(in4, wj, part);
#pragma unroll
                    for (int t = 0; t < TERMS; ++t)
                        *reinterpret_cast<uint4 *>(piece(L::split_at(i, RB == 128 ? 2 * t + v / 8 : t), c, v)) =
                            make_uint4(part[t][0], part[t][1], part[t][2], part[t][3]);
                }
                tc::fence_async_smem();
            }
            tell(&tab->split);
            wait(&tab->got_b, i);
#pragma unroll
            for (int k = 0; k < 128 * (CB / 8) / WORKERS; ++k) {
                const int r = (k * WORKERS + tid) / (CB / 8), v = (k * WORKERS + tid) % (CB / 8);
                const uint4 b = *reinterpret_cast<const uint4 *>(piece(L::kB + v / 8 * L::kPanel, r, v));
                for (uint32_t word : {b.x, b.y, b.z, b.w}) {  // 0 times an infinity or a NaN is a NaN
                    const __nv_bfloat162 two = *reinterpret_cast<const __nv_bfloat162 *>(&word);
                    zeros = __hfma2(two, __float2bfloat162_rn(0.f), zeros);
                }
            }
            if (STATE) tell(&tab->weighted);
            bool reached = true;  // whether this row sees the state in front of the chunk
            if constexpr (!STATE) {
                int bound = rev ? 127 : 0;  // the last step that it sees (backwards: the farthest)
                if (some) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        // flags at steps in front of this one; backwards, at it and behind it
                        const int at = row - 32 * (rev ? 3 - k : k), from = max(at, 0);
                        const uint32_t r = resets[rev ? 3 - k : k];
                        const uint32_t f = rev ? (at > 31 ? 0u : r >> from << from) : (at <= 0 ? 0u : at > 31 ? r : r & ((1u << at) - 1));
                        if (f) {
                            bound = rev ? 32 * (3 - k) + __ffs(f) - 1 : 32 * k + 32 - __clz(f);
                            reached = false;
                        }
                    }
                }
                wait(&tab->bar[0], i);
                if (RB == 64 && PC * wc >= 64) wait(&tab->split, i);  // the other warps have read A, whose place the second half takes
                tc::tc_fence_after();
                // P: row `row`, 32 columns at a time, from PC wc on, one after the other (two side by side do not fit the registers)
#pragma unroll 1
                for (int b0 = 0; b0 < PC; b0 += 32) {
                    const int col = PC * wc + b0;
                    const int panel = x + col / 64 * L::kPanel, v0 = col % 64 / 8;
                    if (rev ? col < 32 * lq : col > 32 * lq) {  // nothing of it is seen, whatever it holds
#pragma unroll
                        for (int v = 0; v < 4; ++v) *reinterpret_cast<uint4 *>(piece(panel, row, v0 + v)) = make_uint4(0, 0, 0, 0);
                        continue;
                    }
                    const float *weight = tab->weight + 127 - row + col;
                    float f[32];
                    tc::tmem_ld32(mine + col, f);
#pragma unroll
                    for (int c = 0; c < 32; ++c) f[c] *= weight[c];
                    if (col == 32 * lq) {  // on the diagonal
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (rev ? c < lane : c > lane) f[c] = 0.f;
                    }
                    if (some) {
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (rev ? col + c > bound : col + c < bound) f[c] = 0.f;
                    }
#pragma unroll
                    for (int c = 0; c < 32; c += 8)
                        *reinterpret_cast<uint4 *>(piece(panel, row, v0 + c / 8)) =
                            make_uint4(pack_bf16x2(f[c], f[c + 1]), pack_bf16x2(f[c + 2], f[c + 3]), pack_bf16x2(f[c + 4], f[c + 5]), pack_bf16x2(f[c + 6], f[c + 7]));
                }
                tc::fence_async_smem();
                tc::tc_fence_before();
                tell(&tab->weighted);
            }
            if (update) {
                wait(&tab->bar[1], i);
                tc::tc_fence_after();
                const float keep = tab->pow[n];
#pragma unroll
                for (int c0 = 0; c0 < H; c0 += G) {
                    float f[G];
                    tmem_get<G>(mine + kK + wc * H + c0, f);
#pragma unroll
                    for (int c = 0; c < G; c += 2) {
                        const float2 p = some ? make_float2(f[c], f[c + 1]) : parts(fma2(pair_of(M[c0 + c], M[c0 + c + 1]), pair_of(keep, keep), pair_of(f[c], f[c + 1])));
                        M[c0 + c] = p.x, M[c0 + c + 1] = p.y;
                    }
                }
                if (!STATE && more) store_m();
            }
            if constexpr (!STATE) {
                wait(&tab->bar[2], i);
                tc::tc_fence_after();
                const float f1 = tab->pow[max(rev ? n - 1 - row : row + 1, 0)];
                const long long at = (long long)(start_of(i) + row) * s.Be + e;
#pragma unroll
                for (int c0 = 0; c0 < H; c0 += G) {
                    float o[G];
                    tmem_get<G>(mine + wc * H + c0, o);
                    if (filled) {
                        float m[G];
                        tmem_get<G>(mine + kO1 + wc * H + c0, m);
                        if (reached) {
#pragma unroll
                            for (int c = 0; c < G; c += 2) {
                                const float2 p = parts(fma2(pair_of(m[c], m[c + 1]), pair_of(f1, f1), pair_of(o[c], o[c + 1])));
                                o[c] = p.x, o[c + 1] = p.y;
                            }
                        }
                    }
#pragma unroll
                    for (int c = 0; c < G; c += 2) {
                        const float2 p = parts(mul2(pair_of(o[c], o[c + 1]), pair_of(s.out_scale, s.out_scale)));
                        o[c] = p.x, o[c + 1] = p.y;
                    }
                    if (s.shared) {
                        float *to = s.shared + (at * s.heads + h) * s.C + wc * H + c0;
                        if (row < n) {
#pragma unroll
                            for (int c = 0; c < G; c += 8)
                                if (wc * H + c0 + c < s.C) store_32_bytes(to + c, o + c);  // whole sectors: a lane's neighbours write other rows
                        }
                    } else {  // through the place of P
#pragma unroll
                        for (int c = 0; c < G; c += 8) {
                            const int v = (wc * H + c0 + c) / 8;
                            *reinterpret_cast<uint4 *>(piece(x + v / 8 * L::kPanel, row, v)) =
                                make_uint4(pack_bf16x2(o[c], o[c + 1]), pack_bf16x2(o[c + 2], o[c + 3]), pack_bf16x2(o[c + 4], o[c + 5]), pack_bf16x2(o[c + 6], o[c + 7]));
                        }
                    }
                }
            }
            tc::fence_async_smem();
            tc::tc_fence_before();
            tell(&tab->emptied);
            filled = true;
        }
        if (!__hbeq2(zeros, __float2bfloat162_rn(0.f))) tab->bad = 1;
        if (STATE && tid == 0) s.seg_reset[(size_t)seg * s.Be * s.heads + eh] = any != 0;
        asm volatile("bar.sync 4, %0;" ::"n"(WORKERS) : "memory");
        if (out_state && !tab->bad) {
            if (RB == 64) {  // the two shares of a row
                float *y = reinterpret_cast<float *>(smem + L::split_at(chunks - 1, 0));
                if (row >= 64) {
#pragma unroll
                    for (int c = 0; c < H; ++c) y[(wc * H + c) * 64 + row - 64] = M[c];
                }
                asm volatile("bar.sync 4, %0;" ::"n"(WORKERS) : "memory");
                if (row < 64) {
#pragma unroll
                    for (int c = 0; c < H; ++c) M[c] += y[(wc * H + c) * 64 + row];
                }
            }
            if (mine_on) {
                float *p = out_state + row * sr + wc * H * sc;
                if (sc == 1) {
#pragma unroll
                    for (int c = 0; c < H; c += 4)
                        if (wc * H + c < s.C) *reinterpret_cast<float4 *>(p + c) = make_float4(M[c], M[c + 1], M[c + 2], M[c + 3]);
                } else {
#pragma unroll
                    for (int c = 0; c < H; ++c)
                        if (wc * H + c < s.C) p[c * sc] = M[c];
                }
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (w == 4 * WG) {
        tc::tc_fence_after();
        tc::tmem_dealloc(tab->slot, L::kCols);
    }
    if (tab->bad) segment_slowly<STATE>(s, reinterpret_cast<float *>(smem), in, out_state, sr, sc, eh, t_lo, t_hi);
}

// What each segment starts from, in place of what it adds, and the state that is left.
__global__ void __launch_bounds__(256) segments_kernel(const __grid_constant__ Sweeps all) {
    grid_wait();
    const Sweep &s = all.s[blockIdx.z];
    const int eh = blockIdx.x, h = eh % s.heads, i = blockIdx.y * 256 + threadIdx.x;  // element r * C + c
    if (i >= s.R * s.C) return;
    const long long at = (i / s.C) * s.stride_r + (i % s.C) * s.stride_c, states = (long long)s.Be * s.heads;
    const float l2 = log2f(s.decay[h]), whole = power(l2, s.seg_len), tail = power(l2, s.T - (s.nseg - 1) * s.seg_len);
    float m = s.m_in ? s.m_in[eh * s.state + at] : 0.f;
    float *p = s.seg + eh * (long long)s.R * s.C + i;
    const long long step = states * s.R * s.C;
    for (int n = 0; n < s.nseg; n += 8) {  // in the sweep's order
        float add[8];
        int reset[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int seg = s.reverse ? s.nseg - 1 - n - k : n + k;
            add[k] = n + k < s.nseg ? p[seg * step] : 0.f;
            reset[k] = n + k < s.nseg ? s.seg_reset[seg * states + eh] : 0;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (n + k >= s.nseg) break;
            const int seg = s.reverse ? s.nseg - 1 - n - k : n + k;
            p[seg * step] = m;
            m = reset[k] ? add[k] : fmaf(seg == s.nseg - 1 ? tail : whole, m, add[k]);
        }
    }
    if (s.m_out) s.m_out[eh * s.state + at] = m;
}

// Gradient of a shared head: the sum of those of its query heads.  Four columns a thread where C has them.
template <typename T>
__global__ void __launch_bounds__(256) shared_sum_kernel(const __grid_constant__ Sweeps all, int share) {
    grid_wait();
    const Sweep &s = all.s[blockIdx.z];
    const int C = s.C, kv_heads = s.heads / share, n = C % 4 == 0 ? 4 : 1, width = kv_heads * C / n;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i / width;
    if (row >= (long long)s.T * s.Be) return;
    const int at = (int)(i % width) * n, g = at / C, c = at % C;
    const float *p = s.shared + (row * kv_heads + g) * share * C + c;
    T *to = static_cast<T *>(s.out) + row * s.ldo + at;
    if (n == 4) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < share; ++k) {
            const float4 f = *reinterpret_cast<const float4 *>(p + k * C);
            v.x += f.x, v.y += f.y, v.z += f.z, v.w += f.w;
        }
        to[0] = from_f32<T>(v.x), to[1] = from_f32<T>(v.y), to[2] = from_f32<T>(v.z), to[3] = from_f32<T>(v.w);
    } else {
        float v = 0.f;
        for (int k = 0; k < share; ++k) v += p[k * C];
        to[0] = from_f32<T>(v);
    }
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

// Segments a sequence is cut into: as many as give the GPU one round of two blocks per SM (64 columns of a head each; the GPU's 148
// SMs as a constant, so that the size of the workspace does not depend on where it is asked for), none but the last
// shorter than 256 steps: a segment's states are made, written, joined and read (8192 steps of 16 x 128 in 8 segments: 37 us, 10 to join
// them, 44 for the outputs from there; step by step and whole 1392).  The blocks of one sweep are counted, also where a call for gradients
// launches three together (2048 steps of 4 x 16 heads of 64: 768 blocks, 2.6 rounds).
constexpr int kSegment = 256;
int segments(const ppo_decay_attention_desc *d, int *len) {
    const long long blocks = (long long)d->Be * d->heads * ppo_cdiv(d->dk > d->dv ? d->dk : d->dv, 64);
    int n = blocks < 2 * 148 ? (int)(2 * 148 / blocks) : 1;
    const int most = ppo_cdiv(d->T, kSegment);
    if (n > most) n = most;
    const int per = ppo_cdiv(ppo_cdiv(d->T, n), 128) * 128;
    *len = per;
    return ppo_cdiv(d->T, per);
}

int check(const ppo_decay_attention_desc *d) {
    if (!d || d->T <= 0 || d->Be <= 0 || d->heads <= 0 || d->kv_heads <= 0 || d->dk <= 0 || d->dv <= 0) return PPO_ERR_INVALID_ARG;
    if (d->dtype != PPO_F32 && d->dtype != PPO_BF16) return PPO_ERR_INVALID_ARG;
    if (!(d->scale > -3.0e38f && d->scale < 3.0e38f)) return PPO_ERR_INVALID_ARG;
    if (d->heads % d->kv_heads != 0) return PPO_ERR_SHAPE;
    if (d->dk > 128 || d->dv > 128) return PPO_ERR_UNSUPPORTED;
    if ((long long)d->T * d->Be > 0x7f000000ll || (long long)d->Be * d->heads > 0x1fffffffll) return PPO_ERR_UNSUPPORTED;
    if (d->ldq < (int64_t)d->heads * d->dk || d->ldk < (int64_t)d->kv_heads * d->dk || d->ldv < (int64_t)d->kv_heads * d->dv ||
        d->ldo < (int64_t)d->heads * d->dv)
        return PPO_ERR_SHAPE;
    return PPO_OK;
}

size_t seg_floats(const ppo_decay_attention_desc *d) {
    int len;
    const int n = segments(d, &len);
    return n > 1 ? (size_t)n * d->Be * d->heads * (d->dk * d->dv + 1) + 7 & ~(size_t)7 : 0;  // with a flag each; in 32 bytes
}
// In 32 bits: gradients of shared heads, of each of their query heads; in whole 32 bytes.
size_t shared_floats(const ppo_decay_attention_desc *d, int width) {
    return d->heads != d->kv_heads ? ((size_t)d->T * d->Be * d->heads * width + 7) & ~(size_t)7 : 0;
}

// The sweeps of a call; those from `later` on wait for the others.
struct Work {
    Sweep s[3];
    int n, later;
};

// fn(sweeps, how many) for the sweeps lo .. hi for which `which` holds.
template <typename W, typename F>
int launch_group(const Work &w, int lo, int hi, W &&which, F &&fn) {
    Sweeps all = {};
    int n = 0;
    for (int i = lo; i < hi; ++i)
        if (which(w.s[i])) all.s[n++] = w.s[i];
    return n ? fn(all, n) : PPO_OK;
}
const auto every = [](const Sweep &) { return true; };

// Blocks along x: as many as the sweep with the most columns has, `cols` of them a block.
unsigned blocks_of(const Sweeps &all, int n, int cols) {
    int most = 0;
    for (int i = 0; i < n; ++i) most = most > all.s[i].C ? most : all.s[i].C;
    return (unsigned)(ppo_cdiv(most, cols) * all.s[0].Be * all.s[0].heads);
}

template <typename T, bool STATE>
int sweep_launch(const Sweeps &all, int n, cudaStream_t st) {
    int rows = 0;
    for (int i = 0; i < n; ++i) rows = rows > all.s[i].R ? rows : all.s[i].R;
    const dim3 grid(blocks_of(all, n, kCols), all.s[0].nseg, n);
    if (rows <= 64) return ppo_launch(sweep_kernel<T, STATE, 8>, grid, dim3(256), 0, st, all);
    if (rows <= 96) return ppo_launch(sweep_kernel<T, STATE, 12>, grid, dim3(256), 0, st, all);
    return ppo_launch(sweep_kernel<T, STATE, 16>, grid, dim3(256), 0, st, all);
}
template <int RB>
int chunk_launch(const Sweeps &all, int n, cudaStream_t st) {
    static PerDevice<bool> allowed;
    PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(chunk_kernel<RB>, ChunkSmem<RB>::kBytes); }));
    return ppo_launch(chunk_kernel<RB>, dim3(blocks_of(all, n, kBlockCols), 1, n), dim3(256), ChunkSmem<RB>::kBytes, st, all);
}
template <int RB>
int short_launch(const Sweeps &all, int n, cudaStream_t st) {
    return ppo_launch(short_kernel<RB>, dim3(blocks_of(all, n, kBlockCols), 1, n), dim3(128), 0, st, all);
}

// Rows of heads as [T][Be][heads][width], boxes of 128 steps and 64 columns of one head.
int tile_map(const Sweep &s, TileMap *m) {
    const int box[4] = {64, 1, 1, 128};
    const auto map = [&](CUtensorMap *to, const void *p, int width, int heads, long long ld) {
        const long long dims[4] = {width, heads, s.Be, s.T}, strides[3] = {2ll * width, 2 * ld, 2 * ld * s.Be};
        return make_map_strided(to, p, 4, dims, strides, box);
    };
    PPO_TRY(map(&m->x, s.x, s.R, s.heads / s.share_x, s.ldx));
    PPO_TRY(map(&m->a, s.a, s.R, s.heads / s.share_a, s.lda));
    PPO_TRY(map(&m->b, s.b, s.C, s.heads / s.share_b, s.ldb));
    return s.shared ? PPO_OK : map(&m->out, s.out, s.C, s.heads, s.ldo);
}
template <int RB, int CB, bool STATE, int TERMS>
int tile_launch_as(const Sweeps &all, int n, cudaStream_t st) {
    using L = TileSmem<RB, CB, STATE, TERMS>;
    static PerDevice<bool> allowed;
    int32_t *status = ppo_device_status_ptr();
    if (!status) return PPO_ERR_CUDA;
    PPO_TRY(ppo_once_per_device(allowed, [] { return ppo_allow_smem(tile_kernel<RB, CB, STATE, TERMS>, L::kBytes); }));
    TileMaps maps = {};
    for (int i = 0; i < n; ++i) PPO_TRY(tile_map(all.s[i], &maps.m[i]));
    return ppo_launch(tile_kernel<RB, CB, STATE, TERMS>, dim3(all.s[0].Be * all.s[0].heads, all.s[0].nseg, n), dim3(tile_threads(RB, CB, STATE)), L::kBytes,
                      st, all, maps, status);
}
// The sweeps lo .. hi of `which`, those of one shape together; exact: whether a sweep hands out a state that it makes here.
template <bool STATE, typename W>
int tile_launch(const Work &w, int lo, int hi, W &&which, cudaStream_t st) {
    const auto exact = [](const Sweep &s) { return s.m_out && (STATE || s.nseg == 1); };
    for (int rows = 64; rows <= 128; rows += 64)
        for (int cols = 64; cols <= 128; cols += 64) {
            bool e = false;
            const auto shape = [&](const Sweep &s) { return which(s) && (s.R <= 64) == (rows == 64) && (s.C <= 64) == (cols == 64); };
            PPO_TRY(launch_group(w, lo, hi, shape, [&](const Sweeps &all, int n) {
                for (int i = 0; i < n; ++i) e = e || exact(all.s[i]);
                if (rows == 64 && cols == 64) return e ? tile_launch_as<64, 64, STATE, 4>(all, n, st) : tile_launch_as<64, 64, STATE, 2>(all, n, st);
                if (rows == 64) return e ? tile_launch_as<64, 128, STATE, 4>(all, n, st) : tile_launch_as<64, 128, STATE, 2>(all, n, st);
                if (cols == 64) return e ? tile_launch_as<128, 64, STATE, 3>(all, n, st) : tile_launch_as<128, 64, STATE, 2>(all, n, st);
                return e ? tile_launch_as<128, 128, STATE, 3>(all, n, st) : tile_launch_as<128, 128, STATE, 2>(all, n, st);
            }));
        }
    return PPO_OK;
}
// Rows of 16-byte vectors, which the tiles' maps reach.
bool chunks_fit(const Sweep &s) {
    const auto rows = [&](const void *p, long long ld) { return ppo_aligned(p, 16) && ld % 8 == 0 && ld * s.Be < 1ll << 38; };
    return s.R % 8 == 0 && s.C % 8 == 0 && rows(s.a, s.lda) && rows(s.b, s.ldb) && rows(s.x, s.ldx) && (s.shared || rows(s.out, s.ldo));
}

// bf16 rows that vectors fit: up to 16 steps, up to 64, more.  64 x 16 heads of 64 x 64, outputs and gradients: 16 steps 22 and 37 us,
// 17 (as a chunk of 64) 31 and 60; 64 steps 43 and 80, 65 (in a tile of 128) 68 and 162.
template <typename T>
int run(const Work &w, cudaStream_t st) {
    bool chunks = std::is_same_v<T, bf16>;
    for (int i = 0; i < w.n; ++i) chunks = chunks && chunks_fit(w.s[i]);
    const Sweep &f = w.s[0];
    if (f.nseg > 1) {
        const auto to_make = [](const Sweep &s) { return !s.seg_made; };
        if (chunks) PPO_TRY(tile_launch<true>(w, 0, w.n, to_make, st));
        else PPO_TRY(launch_group(w, 0, w.n, to_make, [&](const Sweeps &all, int n) { return sweep_launch<T, true>(all, n, st); }));
        PPO_TRY(launch_group(w, 0, w.n, to_make, [&](const Sweeps &all, int n) {
            return ppo_launch(segments_kernel, dim3(f.Be * f.heads, ppo_cdiv(f.R * f.C, 256), n), dim3(256), 0, st, all);
        }));
    }
    for (int lo = 0; lo < w.n; lo = lo < w.later ? w.later : w.n) {
        const int hi = lo < w.later ? w.later : w.n;
        if (!chunks) {
            PPO_TRY(launch_group(w, lo, hi, every, [&](const Sweeps &all, int n) { return sweep_launch<T, false>(all, n, st); }));
        } else if (f.T > kChunk) {
            PPO_TRY(tile_launch<false>(w, lo, hi, every, st));
        } else {
            PPO_TRY(launch_group(w, lo, hi, [](const Sweep &s) { return s.R <= 64; }, [&](const Sweeps &all, int n) {
                return f.T <= 16 ? short_launch<64>(all, n, st) : chunk_launch<64>(all, n, st);
            }));
            PPO_TRY(launch_group(w, lo, hi, [](const Sweep &s) { return s.R > 64; }, [&](const Sweeps &all, int n) {
                return f.T <= 16 ? short_launch<128>(all, n, st) : chunk_launch<128>(all, n, st);
            }));
        }
    }
    return launch_group(w, 0, w.n, [](const Sweep &s) { return s.shared != nullptr; }, [&](const Sweeps &all, int n) {
        const int share = all.s[0].share_x;
        long long most = 0;
        for (int i = 0; i < n; ++i) {
            const long long items = (long long)f.T * f.Be * f.heads / share * all.s[i].C / (all.s[i].C % 4 == 0 ? 4 : 1);
            most = most > items ? most : items;
        }
        return ppo_launch(shared_sum_kernel<T>, dim3((unsigned)((most + 255) / 256), 1, n), dim3(256), 0, st, all, share);
    });
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
    s.seg_reset = reinterpret_cast<int *>(seg + (size_t)s.nseg * d->Be * d->heads * d->dk * d->dv);
    return s;
}
// M [dk][dv], the state as it is stored, or M [dv][dk]
void plain_state(Sweep *s, const ppo_decay_attention_desc *d) {
    s->R = d->dk;
    s->C = d->dv;
    s->stride_r = s->seg_r = d->dv;
    s->stride_c = s->seg_c = 1;
}
void turned_state(Sweep *s, const ppo_decay_attention_desc *d) {
    s->R = d->dv;
    s->C = d->dk;
    s->stride_r = 1;
    s->stride_c = d->dv;
    s->seg_r = d->dk;
    s->seg_c = 1;
}

bool misaligned(std::initializer_list<const void *> ps, size_t a) {
    for (const void *p : ps)
        if (!ppo_aligned(p, a)) return true;
    return false;
}

}  // namespace

extern "C" size_t ppo_decay_attention_workspace_bytes(const ppo_decay_attention_desc *d, int backward) {
    if (check(d) != PPO_OK) return 0;
    if (!backward) return seg_floats(d) * sizeof(float);
    return (2 * seg_floats(d) + shared_floats(d, d->dk) + shared_floats(d, d->dv)) * sizeof(float);
}

extern "C" int ppo_decay_attention_fwd(const ppo_decay_attention_desc *d, const void *q, const void *k, const void *v, const float *decay,
                                       const uint8_t *done, const float *state_in, void *o, float *state_out, void *workspace, size_t ws_bytes,
                                       void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_decay_attention_workspace_bytes(d, 0);
    if (!q || !k || !v || !decay || !o || (need > 0 && !workspace)) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({q, k, v, o}, elem_bytes(d->dtype)) || misaligned({decay}, 4) || misaligned({state_in, state_out}, 16) || misaligned({workspace}, 32)) return PPO_ERR_ALIGN;
    Work w = {};
    w.n = w.later = 1;
    Sweep &s = w.s[0];
    s = sweep_of(d, decay, done, static_cast<float *>(workspace));
    plain_state(&s, d);
    s.a = k, s.lda = d->ldk, s.b = v, s.ldb = d->ldv, s.x = q, s.ldx = d->ldq, s.out = o, s.ldo = d->ldo;
    s.share_a = s.share_b = d->heads / d->kv_heads;
    s.out_scale = d->scale;
    s.m_in = state_in;
    s.m_out = state_out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d->dtype == PPO_F32 ? run<float>(w, st) : run<bf16>(w, st);
}

extern "C" int ppo_decay_attention_bwd(const ppo_decay_attention_desc *d, const void *q, const void *k, const void *v, const float *decay,
                                       const uint8_t *done, const float *state_in, const void *d_o, const float *dstate_out, void *dq, void *dk,
                                       void *dv, float *dstate_in, void *workspace, size_t ws_bytes, void *stream) {
    PPO_TRY(check(d));
    const size_t need = ppo_decay_attention_workspace_bytes(d, 1);
    if (!q || !k || !v || !decay || !d_o || !dq || !dk || !dv || (need > 0 && !workspace)) return PPO_ERR_INVALID_ARG;
    if (ws_bytes < need) return PPO_ERR_SHAPE;
    if (misaligned({q, k, v, d_o, dq, dk, dv}, elem_bytes(d->dtype)) || misaligned({decay}, 4) ||
        misaligned({state_in, dstate_out, dstate_in}, 16) || misaligned({workspace}, 32))
        return PPO_ERR_ALIGN;
    const int share = d->heads / d->kv_heads;
    float *seg = static_cast<float *>(workspace), *back = seg + seg_floats(d), *part = share > 1 ? back + seg_floats(d) : nullptr;
    Work w = {};
    Sweep &sq = w.s[0], &sk = w.s[1], &sv = w.s[2];
    sq = sweep_of(d, decay, done, seg);
    turned_state(&sq, d);
    sq.a = v, sq.lda = d->ldv, sq.b = k, sq.ldb = d->ldk, sq.x = d_o, sq.ldx = d->ldo, sq.out = dq, sq.ldo = d->ldq;
    sq.share_a = sq.share_b = share;
    sq.out_scale = d->scale;
    sq.m_in = state_in;
    sk = sweep_of(d, decay, done, back);
    turned_state(&sk, d);
    sk.a = d_o, sk.lda = d->ldo, sk.b = q, sk.ldb = d->ldq, sk.x = v, sk.ldx = d->ldv, sk.out = dk, sk.ldo = d->ldk;
    sk.shared = part;
    sv = sweep_of(d, decay, done, back);
    plain_state(&sv, d);
    sv.a = q, sv.lda = d->ldq, sv.b = d_o, sv.ldb = d->ldo, sv.x = k, sv.ldx = d->ldk, sv.out = dv, sv.ldo = d->ldv;
    sv.m_out = dstate_in;
    sv.shared = part ? part + shared_floats(d, d->dk) : nullptr;
    for (Sweep *s : {&sk, &sv}) {
        s->reverse = 1;
        s->share_x = share;
        s->m_in = dstate_out;
        s->a_scale = d->scale;
    }
    // with segments dv's states are dk's, turned; without, dv's sweep may overwrite those that dk's starts from
    sk.seg_made = sk.nseg > 1;
    sk.seg_r = 1;
    sk.seg_c = d->dv;
    w.n = 3;
    w.later = sk.nseg == 1 && dstate_in && dstate_in == dstate_out ? 2 : 3;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d->dtype == PPO_F32 ? run<float>(w, st) : run<bf16>(w, st);
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
