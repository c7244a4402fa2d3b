// C entry points of the operators of a training step: arguments are looked at, nothing else.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <new>
#include <utility>
#include <vector>

#include "train_adamw.hpp"
#include "train_blocks.hpp"
#include "train_norm.hpp"
#include "train_plan.hpp"

namespace qsdp_train {
namespace {

constexpr uint64_t kMostRows = 0x7fffffffu, kMostNorm = 1u << 24, kMostWide = 1u << 26, kMostSum = 1u << 20;

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool known(qsdp_dtype t) { return t == QSDP_F32 || t == QSDP_BF16 || t == QSDP_F16; }
size_t width(qsdp_dtype t) { return t == QSDP_F32 ? 4 : 2; }

int status_of(hipError_t e) { return e == hipSuccess ? QSDP_OK : QSDP_ELAUNCH; }

// The distance of the rows of a matrix (one row has none).
bool stride_ok(uint64_t rows, uint64_t n, uint64_t stride) { return rows <= 1 || (stride >= n && stride <= (1ull << 40)); }

bool norm_ok(qsdp_dtype x, qsdp_dtype y, qsdp_dtype w, uint64_t rows, uint64_t n) {
    return known(x) && known(y) && (x == QSDP_F32 || y == x) && (w == QSDP_F32 || w == y) && rows <= kMostRows && n >= 1 &&
           n <= kMostNorm;
}

bool product_ok(uint64_t m, uint64_t n, uint64_t k) {
    return m <= kMostRows && n >= 1 && n <= kMostWide && k >= 1 && k <= kMostSum;
}

uint64_t pitch_of(uint64_t n) { return blocks_of(n) * kWide; }
uint64_t room(uint64_t bytes) { return (bytes + 15) / 16 * 16; }

// Bytes of rounded rows: codes, then scales.
uint64_t rounded_bytes(uint64_t m, uint64_t k) { return m * pitch_of(k) + room(4 * m * blocks_of(k)); }

bool entry_ok(const qsdp_adamw_tensor& t) {
    const bool eight = t.state_bits == 8;
    if ((!eight && t.state_bits != 32) || t.reserved != 0 || t.n > (1ull << 40) || !std::isfinite(t.lr_scale) ||
        !std::isfinite(t.weight_decay) || t.g_dtype < QSDP_F32 || t.g_dtype > QSDP_F16 || (!eight && t.scale))
        return false;
    if (t.x16 && t.x16_dtype != QSDP_BF16 && t.x16_dtype != QSDP_F16) return false;
    if (t.n == 0) return true;
    return t.x && t.g && t.m && t.v && (!eight || t.scale) && aligned(t.x, 4) &&
           aligned(t.g, width(static_cast<qsdp_dtype>(t.g_dtype))) && aligned(t.m, eight ? 8 : 4) &&
           aligned(t.v, eight ? 8 : 4) && aligned(t.scale, 8) && aligned(t.x16, 2);
}

struct Range {
    uintptr_t from, to;
    bool written;
};

// Whether what is written meets anything else.
bool overlap(std::vector<Range>& ranges) {
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t any = 0, written = 0;  // ends of what lies before, of all of it and of what is written
    for (const Range& r : ranges) {
        if (r.from < written || (r.written && r.from < any)) return true;
        any = std::max(any, r.to);
        if (r.written) written = std::max(written, r.to);
    }
    return false;
}

}  // namespace
}  // namespace qsdp_train

using namespace qsdp_train;

extern "C" {

int qsdp_layer_norm(const void* x, qsdp_dtype dtype, uint64_t rows, uint64_t n, uint64_t row_stride, const void* weight,
                    const void* bias, qsdp_dtype w_dtype, float eps, void* y, qsdp_dtype y_dtype, uint64_t y_row_stride,
                    float* stats, void* stream) {
    if (!norm_ok(dtype, y_dtype, w_dtype, rows, n) || !stride_ok(rows, n, row_stride) || !stride_ok(rows, n, y_row_stride) ||
        !(eps >= 0.0f && std::isfinite(eps)))
        return QSDP_EINVAL;
    if (rows == 0) return QSDP_OK;
    if (!x || !y) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(weight, width(w_dtype)) || !aligned(bias, width(w_dtype)) ||
        !aligned(y, width(y_dtype)) || !aligned(stats, 4))
        return QSDP_EALIGN;
    const NormParams p = {x, rows, n, row_stride, weight, bias, w_dtype, eps, y, y_row_stride, stats, 0};
    return status_of(launch_norm(dtype, y_dtype, p, static_cast<hipStream_t>(stream)));
}

size_t qsdp_layer_norm_backward_bytes(uint64_t rows, uint64_t n) {
    if (rows > kMostRows || n < 1 || n > kMostNorm) return 0;
    return norm_workgroups(rows, n) * 2 * n * 4;
}

int qsdp_layer_norm_backward(const void* x, qsdp_dtype dtype, uint64_t rows, uint64_t n, uint64_t row_stride,
                             const void* weight, qsdp_dtype w_dtype, const float* stats, const void* dy, qsdp_dtype dy_dtype,
                             uint64_t dy_row_stride, void* dx, uint64_t dx_row_stride, float* dw, float* db, int accumulate,
                             void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!norm_ok(dtype, dy_dtype, w_dtype, rows, n) || !stride_ok(rows, n, row_stride) || !stride_ok(rows, n, dy_row_stride) ||
        (dx && !stride_ok(rows, n, dx_row_stride)) || (!dx && !dw && !db))
        return QSDP_EINVAL;
    if (rows == 0 && (accumulate || (!dw && !db))) return QSDP_OK;
    if (rows && (!x || !stats || !dy)) return QSDP_EINVAL;
    if (rows && (dw || db) && (!workspace || workspace_bytes < qsdp_layer_norm_backward_bytes(rows, n))) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(weight, width(w_dtype)) || !aligned(stats, 4) || !aligned(dy, width(dy_dtype)) ||
        !aligned(dx, width(dtype)) || !aligned(dw, 4) || !aligned(db, 4) || !aligned(workspace, 16))
        return QSDP_EALIGN;
    const NormBackwardParams p = {x, rows, n, row_stride, weight, w_dtype, stats, dy, dy_row_stride, dx, dx_row_stride,
                                  dw || db ? static_cast<float*>(workspace) : nullptr};
    return status_of(launch_norm_backward(dtype, dy_dtype, p, dw, db, accumulate != 0, static_cast<hipStream_t>(stream)));
}

int qsdp_quantize_blocks(const void* x, qsdp_dtype dtype, uint64_t rows, uint64_t cols, uint64_t row_stride, int square,
                         uint8_t* codes, float* scales, uint8_t* codes_t, float* scales_t, void* stream) {
    if (!known(dtype) || rows > kMostWide || cols < 1 || cols > kMostWide || !stride_ok(rows, cols, row_stride)) return QSDP_EINVAL;
    if (rows == 0) return QSDP_OK;
    if (!x || !codes != !scales || !codes_t != !scales_t || (!codes && !codes_t)) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(codes_t, 16) || !aligned(scales_t, 4))
        return QSDP_EALIGN;
    const BlockParams p = {x, rows, cols, row_stride, codes, scales, codes_t, scales_t, 0};
    return status_of(launch_quantize(dtype, square != 0, p, static_cast<hipStream_t>(stream)));
}

size_t qsdp_matmul_blocks_bytes(uint64_t m, uint64_t n, uint64_t k) {
    if (!product_ok(m, n, k)) return 0;
    const uint64_t parts = choose_parts(m, n, k);
    return parts > 1 ? parts * m * n * sizeof(float) : 0;
}

int qsdp_matmul_blocks(const uint8_t* a, const float* a_scales, uint64_t m, const uint8_t* b, const float* b_scales, int b_square,
                       uint64_t n, uint64_t k, const float* bias, qsdp_dtype out_dtype, void* y, uint64_t y_row_stride,
                       int accumulate, void* workspace, uint64_t workspace_bytes, void* stream) {
    if (!known(out_dtype) || !product_ok(m, n, k) || !stride_ok(m, n, y_row_stride)) return QSDP_EINVAL;
    if (m == 0) return QSDP_OK;
    if (!a || !a_scales || !b || !b_scales || !y) return QSDP_EINVAL;
    if (!aligned(a, 16) || !aligned(a_scales, 4) || !aligned(b, 16) || !aligned(b_scales, 4) || !aligned(bias, 4) ||
        !aligned(y, width(out_dtype)) || !aligned(workspace, 16))
        return QSDP_EALIGN;
    const size_t bytes = qsdp_matmul_blocks_bytes(m, n, k);
    const bool shared = bytes && workspace && workspace_bytes >= bytes;
    const ProductParams p = {a, a_scales, m, m, b, b_scales, n, k, pitch_of(k), bias, out_dtype, y, y_row_stride,
                             accumulate != 0, shared ? static_cast<float*>(workspace) : nullptr, 0, 0};
    return status_of(launch_product(b_square != 0, p, static_cast<hipStream_t>(stream)));
}

size_t qsdp_linear_blocks_bytes(uint64_t m, uint64_t n, uint64_t k) {
    if (!product_ok(m, n, k)) return 0;
    if (m > kFewRows) return rounded_bytes(m, k) + qsdp_matmul_blocks_bytes(m, n, k);
    const uint64_t parts = choose_few_parts(n, k);
    return parts > 1 ? parts * m * n * sizeof(float) : 16;
}

int qsdp_linear_blocks(const void* x, qsdp_dtype dtype, uint64_t m, uint64_t k, uint64_t row_stride, const uint8_t* w,
                       const float* w_scales, uint64_t n, const float* bias, qsdp_dtype out_dtype, void* y,
                       uint64_t y_row_stride, void* workspace, uint64_t workspace_bytes, void* stream) {
    // everything is looked at before the first launch
    if (!known(dtype) || !known(out_dtype) || !product_ok(m, n, k) || m > kMostWide || !stride_ok(m, k, row_stride) ||
        !stride_ok(m, n, y_row_stride))
        return QSDP_EINVAL;
    if (m == 0) return QSDP_OK;
    if (!x || !w || !w_scales || !y || !workspace || workspace_bytes < qsdp_linear_blocks_bytes(m, n, k)) return QSDP_EINVAL;
    if (!aligned(x, width(dtype)) || !aligned(w, 16) || !aligned(w_scales, 4) || !aligned(bias, 4) ||
        !aligned(y, width(out_dtype)) || !aligned(workspace, 16))
        return QSDP_EALIGN;
    if (m <= kFewRows) {
        const ProductParams p = {nullptr, nullptr, m, m, w, w_scales, n, k, pitch_of(k), bias, out_dtype, y, y_row_stride, false,
                                 static_cast<float*>(workspace), 0, 0};
        return status_of(launch_linear_few({x, dtype, row_stride}, p, static_cast<hipStream_t>(stream)));
    }
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    float* scales = reinterpret_cast<float*>(codes + m * pitch_of(k));
    const int status = qsdp_quantize_blocks(x, dtype, m, k, row_stride, 0, codes, scales, nullptr, nullptr, stream);
    if (status != QSDP_OK) return status;
    uint8_t* rest = codes + rounded_bytes(m, k);
    return qsdp_matmul_blocks(codes, scales, m, w, w_scales, 1, n, k, bias, out_dtype, y, y_row_stride, 0, rest,
                              workspace_bytes - rounded_bytes(m, k), stream);
}

uint64_t qsdp_adamw_build(qsdp_adamw_tensor* table, uint32_t count) {
    if (!table) return 0;
    try {
        std::vector<Range> ranges;
        uint64_t pieces = 0;
        for (uint32_t i = 0; i < count; ++i) {
            const qsdp_adamw_tensor& t = table[i];
            if (!entry_ok(t)) return 0;
            if (t.n) {
                auto add = [&](const void* p, uint64_t bytes, bool written) {
                    if (p) ranges.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
                };
                const uint64_t state = t.state_bits == 8 ? 1 : 4;
                add(t.x, 4 * t.n, true);
                add(t.m, state * t.n, true);
                add(t.v, state * t.n, true);
                add(t.scale, 8 * ((t.n + kBlock - 1) / kBlock), true);
                add(t.x16, 2 * t.n, true);
                add(t.g, width(static_cast<qsdp_dtype>(t.g_dtype)) * t.n, false);
            }
            pieces += (t.n + kPiece - 1) / kPiece;
        }
        if (overlap(ranges)) return 0;
        uint64_t first = 0;
        for (uint32_t i = 0; i < count; ++i) {
            table[i].first = first;
            first += (table[i].n + kPiece - 1) / kPiece;
        }
        return pieces;
    } catch (const std::bad_alloc&) {
        return 0;
    }
}

int qsdp_adamw_tensors(const qsdp_adamw_tensor* table, uint32_t count, uint64_t pieces, float lr, float beta1, float beta2,
                       float eps, float bias1, float bias2, uint64_t seed, const uint64_t* seed_dev, const float* schedule,
                       const float* grad_scale, void* stream) {
    if (!table || count == 0 || pieces == 0 || !std::isfinite(lr) || !(beta1 >= 0.0f && beta1 < 1.0f) ||
        !(beta2 >= 0.0f && beta2 < 1.0f) || !(eps >= 0x1p-126f && std::isfinite(eps)) || !(bias1 > 0.0f && std::isfinite(bias1)) ||
        !(bias2 > 0.0f && std::isfinite(bias2)))
        return QSDP_EINVAL;
    if (!aligned(table, 8) || !aligned(seed_dev, 8) || !aligned(schedule, 4) || !aligned(grad_scale, 4)) return QSDP_EALIGN;
    const AdamWParams p = {table, count, 0, lr, beta1, beta2, eps, 1.0f / bias1, 1.0f / std::sqrt(bias2), seed, seed_dev, schedule,
                           grad_scale};
    return status_of(launch_adamw(p, pieces, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
