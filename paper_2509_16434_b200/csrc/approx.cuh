// Exponentials, sigmoids and their relatives from the hardware's approximations, each within a few units of the last of 24 bits; results below
// 2^-126 are 0.
#pragma once

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
    return fmaf(2.f * s, p, v > 0.f ? v : v == v ? 0.f : v);
}
