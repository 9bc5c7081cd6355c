// Internal launch interface between the C ABI (api.hip) and the kernels of group norm and dropout (norm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace nerva {

// What is dropped: `cut` of 65536 entries on average, those that are kept are multiplied by `scale`.
struct DropArgs {
    uint32_t cut;            // 0: nothing
    float scale;             // 65536 / (65536 - cut)
    uint32_t layer;
    const int64_t *state;    // {seed, step} on the device; not read where cut is 0
};

struct NormArgs {
    const float *X;
    int64_t ldx;
    const float *gamma, *beta;       // [features] or nullptr
    int32_t features, groups, batch, act;
    float eps;
    DropArgs drop;
    float *Y;                        // forward
    int64_t ldy;
    float *mean, *rstd;              // (groups, lds); written by the forward pass unless nullptr, read by the backward pass
    int64_t lds;
    const float *dY;                 // backward
    int64_t lddy;
    float *dX;
    int64_t lddx;
    float *dgamma, *dbeta;           // or nullptr
    float *workspace;
};
// floats of scratch memory that either pass of these sizes takes
int64_t norm_scratch_floats(int32_t features, int32_t groups, int32_t batch);
// hipErrorInvalidConfiguration, with nothing launched, where a launch would take more threads than there may be
hipError_t launch_norm_forward(const NormArgs &a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs &a, hipStream_t s);

struct DropoutArgs {
    const float *X;
    int64_t ldx;
    float *Y;
    int64_t ldy;
    int32_t features, batch;
    DropArgs drop;
};
hipError_t launch_dropout(const DropoutArgs &a, hipStream_t s);

}  // namespace nerva
