// Parameters of the product of rounded tokens with packed weights (lm_linear.hip), filled by the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_lm {

struct TokenParams {
    const void* x;
    uint64_t rows, k, stride;  // elements
    uint32_t bucket, buckets;  // of a row
    int8_t* codes;
    uint64_t pitch;  // bytes from a token's codes to the next one's
    float *scale, *sums;
    uint64_t first;  // token of a launch's first workgroup
};

struct MatmulParams {
    const int8_t* x;
    uint64_t x_pitch;
    const float *x_scale, *x_sums;
    uint64_t m;
    const uint8_t* w;
    uint64_t w_pitch;  // bytes of a channel's codes: whole buckets
    const float* meta;
    uint64_t n, k;
    uint32_t bucket, buckets;
    const float* bias;
    void* y;
    uint64_t y_stride;  // elements
};

hipError_t launch_tokens(qsdp_dtype dtype, const TokenParams& p, hipStream_t s);
hipError_t launch_matmul(qsdp_dtype out, const MatmulParams& p, hipStream_t s);

}  // namespace qsdp_lm
