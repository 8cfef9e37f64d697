// Arguments of the sampling kernels.
#pragma once

#include <hip/hip_runtime.h>

struct SampleArgs {
    const void* scores;
    long long row;
    int rows, n;
    int shift;                 // a weight's unit is 2^-shift
    int parts, part_len;       // workgroups of a row, and scores of one
    char* scratch;
    const float* u;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    int* token;
    float* logprob;
};

int sample_parts(int rows, int n);
// scratch for calls of up to so many rows and scores
size_t sample_scratch(int rows, int n);
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s);
