// Internal interface between the host side of what an engine's iteration does
// around its attention (step_api.cpp) and the kernels (norm.hip, sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tl {

struct NormParams {
    int64_t n_rows;
    int32_t n_cols;
    int32_t dtype;                  // TL_BF16, TL_F16 or TL_F32
    int32_t group;                  // -1: output in dtype, 0: e4m3 with a scale a row, else columns of a scale
    float eps;
    const void* x;
    const void* residual;           // nullable
    const void* weight;
    int64_t x_stride, residual_stride;      // elements between rows
    void* out;
    float* scale;
    void* sum;                      // nullable
};

struct SampleParams {
    int64_t n_rows, stride;         // elements between rows
    int32_t n_cols;
    int32_t dtype;
    const void* logits;
    const float* u;
    const float* temperature;       // these four are nullable
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    int32_t* token;
    float* logprob;                 // nullable
};

hipError_t launch_norm(const NormParams& p, hipStream_t stream);
hipError_t launch_sample(const SampleParams& p, hipStream_t stream);

}  // namespace tl
