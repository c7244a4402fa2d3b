// Parameters of the AdamW step over many tensors (train_adamw.hip), filled by the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_train {

constexpr uint32_t kBlock = 256;  // elements that share a scale where moments have 8 bits
constexpr uint32_t kPiece = 2048;  // elements of a workgroup, of one tensor

struct AdamWParams {
    const qsdp_adamw_tensor* table;
    uint32_t count;
    uint64_t first;  // piece of a launch's first workgroup
    float lr, beta1, beta2, eps, inverse1, inverse2;  // 1 / bias1, 1 / sqrt(bias2)
    uint64_t seed;
    const uint64_t* seed_increment;  // or none
    const float *schedule, *grad_scale;  // or none
};

hipError_t launch_adamw(AdamWParams p, uint64_t pieces, hipStream_t s);

}  // namespace qsdp_train
