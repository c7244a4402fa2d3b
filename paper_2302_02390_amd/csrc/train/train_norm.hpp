// Parameters of layer norm's kernels (train_norm.hip), filled by the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_train {

struct NormParams {
    const void* x;
    uint64_t rows, n, x_stride;  // elements
    const void *weight, *bias;   // or none
    qsdp_dtype w_dtype;
    float eps;
    void* y;
    uint64_t y_stride;
    float* stats;  // {mean, 1 / standard deviation} of each row, or none
    uint64_t first;  // row of a launch's first workgroup
};

struct NormBackwardParams {
    const void* x;
    uint64_t rows, n, x_stride;
    const void* weight;
    qsdp_dtype w_dtype;
    const float* stats;
    const void* dy;
    uint64_t dy_stride;
    void* dx;  // or none
    uint64_t dx_stride;
    float* partial;  // [workgroups, 2, n]: sums over a workgroup's rows
};

hipError_t launch_norm(qsdp_dtype x, qsdp_dtype y, NormParams p, hipStream_t s);
// Sums over all rows go to dw and db (either may be NULL), on top of what they hold where `accumulate`.
hipError_t launch_norm_backward(qsdp_dtype x, qsdp_dtype y, const NormBackwardParams& p, float* dw, float* db, bool accumulate,
                                hipStream_t s);

}  // namespace qsdp_train
