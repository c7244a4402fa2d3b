// C entry points of the operators on logits and on packed weights: arguments are looked at, nothing else.
#include <cmath>
#include <type_traits>

#include "lm_linear.hpp"
#include "lm_rows.hpp"

namespace qsdp_lm {
namespace {

constexpr uint64_t kMost = 0x7fffffffu;  // rows, vocabulary, tokens, channels
constexpr int kMostTop = 128;

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool known(qsdp_dtype t) { return t == QSDP_F32 || t == QSDP_BF16 || t == QSDP_F16; }
size_t width(qsdp_dtype t) { return t == QSDP_F32 ? 4 : 2; }

// f with a null pointer to the format's type.
template <class F>
hipError_t by_format(qsdp_dtype t, F f) {
    return t == QSDP_F32 ? f((F32*)nullptr) : t == QSDP_BF16 ? f((BF16*)nullptr) : f((F16*)nullptr);
}

int status_of(hipError_t e) { return e == hipSuccess ? QSDP_OK : QSDP_ELAUNCH; }

// A matrix of rows of `n` elements, `stride` apart (one row has none).
bool rows_ok(uint64_t rows, uint64_t n, uint64_t stride) {
    return rows <= kMost && n >= 1 && n <= kMost && (rows <= 1 || (stride >= n && stride <= (1ull << 40)));
}

bool logits_ok(qsdp_dtype dtype, uint64_t rows, uint64_t vocab, uint64_t stride, float temperature) {
    return known(dtype) && rows_ok(rows, vocab, stride) && temperature > 0.0f && std::isfinite(temperature) &&
           std::isfinite(1.0f / temperature);
}

bool distill_ok(int top, float alpha, const void* index, const void* logit, const void* labels) {
    return top >= 0 && top <= kMostTop && alpha >= 0.0f && alpha <= 1.0f && (alpha == 0.0f || top >= 1) &&
           (top == 0 || (index && logit)) && (alpha == 1.0f || labels);
}

// Entries of a list of no weight are not read: what they hold would come into the gradient as a NaN.
int looked_at(int top, float alpha) { return alpha > 0.0f ? top : 0; }

// A channel is one bucket, or several buckets of whole steps of the product. (2^26 channels of 2^20 codes: 64 TB.)
bool product_ok(uint64_t m, uint64_t n, uint64_t k, int bucket) {
    return m <= kMost && n >= 1 && n <= (1u << 26) && k >= 1 && k <= (1u << 20) && bucket >= 32 && bucket <= 8192 &&
           bucket % 32 == 0 && (k <= (uint64_t)bucket || bucket % 128 == 0);
}

uint64_t token_pitch(uint64_t k) { return (k + 127) / 128 * 128; }
uint64_t buckets_of(uint64_t k, int bucket) { return (k + (uint64_t)bucket - 1) / (uint64_t)bucket; }

}  // namespace
}  // namespace qsdp_lm

using namespace qsdp_lm;

extern "C" {

size_t qsdp_token_logprobs_bytes(uint64_t rows, uint64_t vocab, int top) {
    return top < 0 || top > kMostTop ? 0 : parts_bytes(rows, vocab, top);
}

int qsdp_token_logprobs(const void* logits, qsdp_dtype dtype, uint64_t rows, uint64_t vocab, uint64_t row_stride,
                        const int64_t* tokens, float temperature, int top, float* logprob, float* entropy, float* stats,
                        float* top_logprob, int32_t* top_index, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!logits_ok(dtype, rows, vocab, row_stride, temperature) || top < 0 || top > kMostTop || (uint64_t)top > vocab)
        return QSDP_EINVAL;
    if (rows == 0) return QSDP_OK;
    if (!logits || (logprob && !tokens) || (top > 0 && (!top_logprob || !top_index)) ||
        (!logprob && !entropy && !stats && top == 0))
        return QSDP_EINVAL;
    if (!aligned(logits, width(dtype)) || !aligned(tokens, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
        !aligned(stats, 4) || !aligned(top_logprob, 4) || !aligned(top_index, 4) || !aligned(workspace, 16))
        return QSDP_EALIGN;
    ScoreParams p = {{logits, rows, vocab, row_stride, 1.0f / temperature, 0}, tokens, top, logprob, entropy, stats,
                     top_logprob, top_index, 0, nullptr, nullptr};
    const uint64_t parts = parts_bytes(rows, vocab, top);
    if (workspace && parts && workspace_bytes >= parts) {
        p.per = ((vocab + kParts - 1) / kParts + 7) / 8 * 8;  // the last part has at least a seventh of that, and the top
        p.heads = static_cast<float4*>(workspace);
        p.keys = reinterpret_cast<uint64_t*>(p.heads + rows * kParts);
    }
    return status_of(by_format(dtype, [&](auto* t) {
        return launch_score<std::remove_pointer_t<decltype(t)>>(p, static_cast<hipStream_t>(stream));
    }));
}

int qsdp_token_logprobs_backward(const void* logits, qsdp_dtype dtype, uint64_t rows, uint64_t vocab, uint64_t row_stride,
                                 const int64_t* tokens, float temperature, const float* stats, const float* entropy,
                                 const float* d_logprob, const float* d_entropy, void* d_logits, uint64_t d_row_stride,
                                 void* stream) {
    if (!logits_ok(dtype, rows, vocab, row_stride, temperature) || !rows_ok(rows, vocab, d_row_stride)) return QSDP_EINVAL;
    if (rows == 0) return QSDP_OK;
    if (!logits || !stats || !d_logits || (d_logprob && !tokens) || (d_entropy && !entropy) || (!d_logprob && !d_entropy))
        return QSDP_EINVAL;
    if (!aligned(logits, width(dtype)) || !aligned(tokens, 8) || !aligned(stats, 4) || !aligned(entropy, 4) ||
        !aligned(d_logprob, 4) || !aligned(d_entropy, 4) || !aligned(d_logits, width(dtype)))
        return QSDP_EALIGN;
    const ScoreBackwardParams p = {{logits, rows, vocab, row_stride, 1.0f / temperature, 0}, tokens, stats, entropy,
                                   d_logprob, d_entropy, d_logits, d_row_stride};
    return status_of(by_format(dtype, [&](auto* t) {
        return launch_score_backward<std::remove_pointer_t<decltype(t)>>(p, static_cast<hipStream_t>(stream));
    }));
}

int qsdp_distill_loss(const void* logits, qsdp_dtype dtype, uint64_t rows, uint64_t vocab, uint64_t row_stride,
                      const int32_t* teacher_index, const float* teacher_logit, int top, const int64_t* labels,
                      float temperature, float alpha, const float* row_scale, float* loss, float* stats, void* d_logits,
                      uint64_t d_row_stride, void* stream) {
    if (!logits_ok(dtype, rows, vocab, row_stride, temperature) || (d_logits && !rows_ok(rows, vocab, d_row_stride)))
        return QSDP_EINVAL;
    if (rows == 0) return top < 0 || top > kMostTop || !(alpha >= 0.0f && alpha <= 1.0f) ? QSDP_EINVAL : QSDP_OK;
    if (!distill_ok(top, alpha, teacher_index, teacher_logit, labels) || !logits || !loss) return QSDP_EINVAL;
    if (!aligned(logits, width(dtype)) || !aligned(teacher_index, 4) || !aligned(teacher_logit, 4) || !aligned(labels, 8) ||
        !aligned(row_scale, 4) || !aligned(loss, 4) || !aligned(stats, 4) || !aligned(d_logits, width(dtype)))
        return QSDP_EALIGN;
    const DistillParams p = {{logits, rows, vocab, row_stride, 1.0f / temperature, 0}, teacher_index, teacher_logit,
                             looked_at(top, alpha), labels, temperature, alpha, row_scale, nullptr, loss, stats, d_logits,
                             d_row_stride};
    return status_of(by_format(dtype, [&](auto* t) {
        return launch_distill<std::remove_pointer_t<decltype(t)>>(p, static_cast<hipStream_t>(stream));
    }));
}

int qsdp_distill_loss_backward(const void* logits, qsdp_dtype dtype, uint64_t rows, uint64_t vocab, uint64_t row_stride,
                               const int32_t* teacher_index, const float* teacher_logit, int top, const int64_t* labels,
                               float temperature, float alpha, const float* stats, const float* d_loss, void* d_logits,
                               uint64_t d_row_stride, void* stream) {
    if (!logits_ok(dtype, rows, vocab, row_stride, temperature) || !rows_ok(rows, vocab, d_row_stride)) return QSDP_EINVAL;
    if (rows == 0) return top < 0 || top > kMostTop || !(alpha >= 0.0f && alpha <= 1.0f) ? QSDP_EINVAL : QSDP_OK;
    if (!distill_ok(top, alpha, teacher_index, teacher_logit, labels) || !logits || !stats || !d_loss || !d_logits)
        return QSDP_EINVAL;
    if (!aligned(logits, width(dtype)) || !aligned(teacher_index, 4) || !aligned(teacher_logit, 4) || !aligned(labels, 8) ||
        !aligned(stats, 4) || !aligned(d_loss, 4) || !aligned(d_logits, width(dtype)))
        return QSDP_EALIGN;
    const DistillParams p = {{logits, rows, vocab, row_stride, 1.0f / temperature, 0}, teacher_index, teacher_logit,
                             looked_at(top, alpha), labels, temperature, alpha, nullptr, d_loss, nullptr,
                             const_cast<float*>(stats), d_logits, d_row_stride};
    return status_of(by_format(dtype, [&](auto* t) {
        return launch_distill<std::remove_pointer_t<decltype(t)>>(p, static_cast<hipStream_t>(stream));
    }));
}

int qsdp_quantize_tokens(const void* x, qsdp_dtype dtype, uint64_t m, uint64_t k, uint64_t row_stride, int bucket,
                         int8_t* codes, float* scale, float* sums, void* stream) {
    if (!known(dtype) || !product_ok(m, 1, k, bucket) || !rows_ok(m, k, row_stride)) return QSDP_EINVAL;
    if (m == 0) return QSDP_OK;
    if (!x || !codes || !scale || !sums) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(codes, 16) || !aligned(scale, 4) || !aligned(sums, 4)) return QSDP_EALIGN;
    const TokenParams p = {x, m, k, row_stride, (uint32_t)bucket, (uint32_t)buckets_of(k, bucket), codes, token_pitch(k),
                           scale, sums, 0};
    return status_of(launch_tokens(dtype, p, static_cast<hipStream_t>(stream)));
}

int qsdp_matmul_codes(const int8_t* codes, const float* scale, const float* sums, uint64_t m, const uint32_t* wcodes,
                      const float* wmeta, uint64_t n, uint64_t k, int bucket, const float* bias, qsdp_dtype out_dtype,
                      void* y, uint64_t y_row_stride, void* stream) {
    if (!known(out_dtype) || !product_ok(m, n, k, bucket) || !rows_ok(m, n, y_row_stride)) return QSDP_EINVAL;
    if (m == 0) return QSDP_OK;
    if (!codes || !scale || !sums || !wcodes || !wmeta || !y) return QSDP_EINVAL;
    if (!aligned(codes, 16) || !aligned(scale, 4) || !aligned(sums, 4) || !aligned(wcodes, 16) || !aligned(wmeta, 8) ||
        !aligned(bias, 4) || !aligned(y, width(out_dtype)))
        return QSDP_EALIGN;
    const uint64_t buckets = buckets_of(k, bucket);
    const MatmulParams p = {codes, token_pitch(k), scale, sums, m, reinterpret_cast<const uint8_t*>(wcodes),
                            buckets * (uint64_t)bucket, wmeta, n, k, (uint32_t)bucket, (uint32_t)buckets, bias, y,
                            y_row_stride};
    return status_of(launch_matmul(out_dtype, p, static_cast<hipStream_t>(stream)));
}

size_t qsdp_tokens_bytes(uint64_t m, uint64_t k, int bucket) {
    if (!product_ok(m, 1, k, bucket)) return 0;
    return m * (token_pitch(k) + 4 + 4 * buckets_of(k, bucket));
}

int qsdp_linear_codes(const void* x, qsdp_dtype dtype, uint64_t m, uint64_t k, uint64_t row_stride, const uint32_t* wcodes,
                      const float* wmeta, uint64_t n, int bucket, const float* bias, qsdp_dtype out_dtype, void* y,
                      uint64_t y_row_stride, void* workspace, uint64_t workspace_bytes, void* stream) {
    // everything is looked at before the first launch
    if (!known(dtype) || !known(out_dtype) || !product_ok(m, n, k, bucket) || !rows_ok(m, k, row_stride) ||
        !rows_ok(m, n, y_row_stride))
        return QSDP_EINVAL;
    if (m == 0) return QSDP_OK;
    if (!x || !wcodes || !wmeta || !y || !workspace || workspace_bytes < qsdp_tokens_bytes(m, k, bucket)) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(wcodes, 16) || !aligned(wmeta, 8) || !aligned(bias, 4) ||
        !aligned(y, width(out_dtype)) || !aligned(workspace, 16))
        return QSDP_EALIGN;
    int8_t* codes = static_cast<int8_t*>(workspace);
    float* scale = reinterpret_cast<float*>(codes + m * token_pitch(k));
    const int status = qsdp_quantize_tokens(x, dtype, m, k, row_stride, bucket, codes, scale, scale + m, stream);
    if (status != QSDP_OK) return status;
    return qsdp_matmul_codes(codes, scale, scale + m, m, wcodes, wmeta, n, k, bucket, bias, out_dtype, y, y_row_stride,
                             stream);
}

}  // extern "C"
