// Parameters of the kernels on rows of logits (lm_rows.hip), filled by the C entry points (lm_api.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_lm {

struct Rows {
    const void* logits;
    uint64_t rows, vocab, stride;  // elements
    float inv_temperature;
    uint64_t first;  // item of a launch's first workgroup
};

struct ScoreParams {
    Rows in;
    const int64_t* tokens;
    int top;
    float *logprob, *entropy, *stats, *top_logprob;
    int32_t* top_index;
};

struct ScoreBackwardParams {
    Rows in;
    const int64_t* tokens;
    const float *stats, *entropy, *d_logprob, *d_entropy;
    void* d_logits;
    uint64_t d_stride;
};

struct DistillParams {
    Rows in;
    const int32_t* teacher_index;
    const float* teacher_logit;
    int top;
    const int64_t* labels;
    float temperature, alpha;
    const float *row_scale, *d_loss;  // what the gradient is multiplied with: row_scale of a pass that computes the loss, d_loss after it
    float *loss, *stats;              // stats: written with the loss, read by the gradient alone
    void* d_logits;
    uint64_t d_stride;
};

hipError_t launch_score(qsdp_dtype dtype, const ScoreParams& p, hipStream_t s);
hipError_t launch_score_backward(qsdp_dtype dtype, const ScoreBackwardParams& p, hipStream_t s);
hipError_t launch_distill(qsdp_dtype dtype, const DistillParams& p, hipStream_t s);

}  // namespace qsdp_lm
