// Sums of the shares that blocks leave of the gradients of parameters.
#pragma once
#include "launch.cuh"

// Neighbouring stretches of a share and where their sums go (null: not wanted).
struct ParamSums {
    float *out[3];
    long long n[3];
};
// part [parts][n0 + n1 + n2]: written or added to the outputs; in 64 bits and in an order fixed by the sizes.
int ppo_param_sum(const float *part, int parts, const ParamSums &s, int accumulate, cudaStream_t st);
