// Exponentials, sigmoids and their relatives from the hardware's approximations, within a few units of the last of 24 bits, and |z| more of them where
// an argument z is multiplied by log2(e) in front, which rounds it (sigmoids of z far below 0, and softplus there); results below 2^-126 are 0.
#pragma once
#include "pair32.cuh"

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sigmoid_fast(float z) { return rcp_fast(1.f + exp2_fast(-z * kLog2e)); }
// max(v, 0); a NaN stays.
__device__ __forceinline__ float positive(float v) {
    float y;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(v));
    return y;
}
// log(1 + exp(v)) = max(v, 0) + log(1 + e) with e = exp(-|v|), and log(1 + e) = 2 artanh(e / (2 + e)): the argument is at most 1/3, where the
// series up to its 15th power is off by 2^-26.
__device__ __forceinline__ float softplus_fast(float v) {
    const float e = exp2_fast(-fabsf(v) * kLog2e), s = e * rcp_fast(2.f + e), q = s * s;
    float p = fmaf(q, 1.f / 15, 1.f / 13);
    p = fmaf(q, p, 1.f / 11);
    p = fmaf(q, p, 1.f / 9);
    p = fmaf(q, p, 1.f / 7);
    p = fmaf(q, p, 1.f / 5);
    p = fmaf(q, p, 1.f / 3);
    p = fmaf(q, p, 1.f);
    return fmaf(2.f * s, p, positive(v));
}

// The same of two numbers.
__device__ __forceinline__ pair32 twice(float a) { return pair_of(a, a); }
__device__ __forceinline__ pair32 exp2_pair(pair32 p) {
    const float2 f = parts(p);
    return pair_of(exp2_fast(f.x), exp2_fast(f.y));
}
__device__ __forceinline__ pair32 rcp_pair(pair32 p) {
    const float2 f = parts(p);
    return pair_of(rcp_fast(f.x), rcp_fast(f.y));
}
__device__ __forceinline__ pair32 sigmoid_pair(pair32 z) { return rcp_pair(add2(exp2_pair(mul2(z, twice(-kLog2e))), twice(1.f))); }
__device__ __forceinline__ pair32 softplus_pair(pair32 v) {
    const float2 f = parts(v);
    const pair32 e = exp2_pair(mul2(pair_of(fabsf(f.x), fabsf(f.y)), twice(-kLog2e))), s = mul2(e, rcp_pair(add2(e, twice(2.f)))), q = mul2(s, s);
    pair32 p = fma2(q, twice(1.f / 15), twice(1.f / 13));
    p = fma2(q, p, twice(1.f / 11));
    p = fma2(q, p, twice(1.f / 9));
    p = fma2(q, p, twice(1.f / 7));
    p = fma2(q, p, twice(1.f / 5));
    p = fma2(q, p, twice(1.f / 3));
    p = fma2(q, p, twice(1.f));
    return fma2(add2(s, s), p, pair_of(positive(f.x), positive(f.y)));
}
