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
    // Rows shared among workgroups: each takes `per` elements (the last one what is left) and leaves its sums and its first
    // alternatives, [rows, kParts] and [rows, kParts, top].
    uint64_t per;
    float4* heads;
    uint64_t* keys;
};

// Few rows are cut into eight parts where they are long: the bytes of workspace that takes, 0 for other calls. From 65536
// logits on it pays (us without / with, 20 alternatives: one row of 65536 bf16 12 / 11, of 131072 19 / 12, of 262144 float 43 /
// 13; 64 of 65536 12.7 / 12.7, of 131072 21 / 15); below, the second launch costs more than a workgroup alone (50257: 10.2 / 10.8).
constexpr uint64_t kParts = 8;
inline uint64_t parts_bytes(uint64_t rows, uint64_t vocab, int top) {
    return rows <= 64 && vocab >= 65536 ? rows * kParts * (sizeof(float4) + sizeof(uint64_t) * (uint64_t)top) : 0;
}

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

// T: a format of lm_common.hpp.
struct F32;
struct BF16;
struct F16;
template <class T>
hipError_t launch_score(const ScoreParams& p, hipStream_t s);
template <class T>
hipError_t launch_score_backward(const ScoreBackwardParams& p, hipStream_t s);
template <class T>
hipError_t launch_distill(const DistillParams& p, hipStream_t s);

}  // namespace qsdp_lm
