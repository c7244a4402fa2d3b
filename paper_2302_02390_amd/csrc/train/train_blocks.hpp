// Parameters of the rounding to 8-bit floating point in blocks and of products in it (train_blocks.hip, train_product.hip),
// filled by the C entry points.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../../include/qsdp.h"

namespace qsdp_train {

constexpr uint32_t kWide = 128;  // elements of a block along the summed axis, and rows of a square one

constexpr uint64_t blocks_of(uint64_t n) { return (n + kWide - 1) / kWide; }

constexpr float kMostCode = 448.0f, kLeastBlock = 0x1p-100f;

struct BlockParams {
    const void* x;
    uint64_t rows, cols, stride;  // elements
    uint8_t* codes;               // [rows, pitch], or none
    float* scales;                // [blocks of cols, rows or blocks of rows]
    uint8_t* codes_t;             // [cols, pitch of rows], or none
    float* scales_t;              // [blocks of rows, cols or blocks of cols]
    uint64_t first;               // row of tiles of a launch's first workgroup
};

struct ProductParams {
    const uint8_t* a;
    const float* a_scale;  // [blocks, a_rows]
    uint64_t m, a_rows;
    const uint8_t* b;
    const float* b_scale;  // [blocks, blocks of n] or [blocks, n]
    uint64_t n, k, pitch;  // bytes of a row of either operand: whole blocks
    const float* bias;     // or none
    qsdp_dtype out;
    void* y;
    uint64_t y_stride;  // elements
    bool accumulate;
    float* parts;  // workspace for the sums of parts of k, or none
    uint32_t part_steps;
    uint64_t part_elements;  // of a part's sums; both are the launch's
};

// Few rows of a product, as they come: rounded on the way, by every workgroup.
struct FewRows {
    const void* x;
    qsdp_dtype dtype;
    uint64_t stride;  // elements
};

hipError_t launch_quantize(qsdp_dtype dtype, bool square, const BlockParams& p, hipStream_t s);
hipError_t launch_product(bool b_square, const ProductParams& p, hipStream_t s);
// The product of at most kFewRows rows with square blocks; p.a, p.a_scale and p.a_rows are not looked at.
hipError_t launch_linear_few(const FewRows& x, const ProductParams& p, hipStream_t s);

}  // namespace qsdp_train
