// Arguments of the sampling kernels.
#pragma once

#include <hip/hip_runtime.h>

struct SampleArgs {
    const void* scores;
    long long row;
    int rows, n;
    int shift;                 // a weight's unit is 2^-shift
    const float* u;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    int* token;
    float* logprob;
};

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s);
