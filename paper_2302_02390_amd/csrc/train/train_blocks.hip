// Rounding to 8-bit floating point (e4m3: four bits of exponent, three of mantissa, up to 448) with a scale for each block.
//
//   a = max(max |x|, 2^-100) over the block, code = e4m3(x (448 / a)) to nearest even, scale = a / 448
// A block is 128 elements of a row (and of a column, for the transposed codes), or 128 x 128. Operations are binary32, quotients
// IEEE divisions. A NaN stays one. A block with an infinity has an infinite scale and codes 0 (NaN for the infinity): all that is
// summed over it is NaN.
#include "train_blocks.hpp"
#include "train_common.hpp"

namespace qsdp_train {
namespace {

// A workgroup rounds 128 x 128 elements both ways round from one read: a thread has eight consecutive columns of eight
// consecutive rows, so that a row's block is 16 neighbouring lanes, and eight codes of a column, like those of a row, are one store.
template <class T, bool SQUARE>
__global__ __launch_bounds__(256) void quantize_kernel(BlockParams p) {
    __shared__ float largest[4][kWide];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, col = threadIdx.x % 16 * 8, row = threadIdx.x / 16 * 8;
    const uint64_t row_block = p.first + blockIdx.y, col_block = blockIdx.x;
    const uint64_t r0 = row_block * kWide + row, c0 = col_block * kWide + col;
    Raw8<T> raw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (r0 + i < p.rows && c0 < p.cols) raw[i].load(static_cast<const typename T::raw*>(p.x) + (r0 + i) * p.stride + c0, (int)(p.cols - c0));
        else raw[i].none();
    }
    float by_row[8], by_col[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        by_row[i] = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = fabsf(raw[i].at(e));
            by_row[i] = fmaxf(by_row[i], v);
            by_col[e] = i ? fmaxf(by_col[e], v) : v;
        }
    }
    if constexpr (SQUARE) {
        float most = by_row[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) most = fmaxf(most, by_row[i]);
        most = fmaxf(reduce_block<256>(most, Max(), &largest[0][0]), kLeastBlock);
#pragma unroll
        for (int i = 0; i < 8; ++i) by_row[i] = by_col[i] = most;
        if (threadIdx.x == 0) {
            if (p.codes) p.scales[col_block * blocks_of(p.rows) + row_block] = most / kMostCode;
            if (p.codes_t) p.scales_t[row_block * blocks_of(p.cols) + col_block] = most / kMostCode;
        }
    } else {
        if (p.codes) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                by_row[i] = fmaxf(reduce16(by_row[i], Max()), kLeastBlock);
                if (lane % 16 == i && r0 + i < p.rows) p.scales[col_block * p.rows + r0 + i] = by_row[i] / kMostCode;
            }
        }
        if (p.codes_t) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                by_col[e] = largest_of_rows(by_col[e]);
                if (lane < 16) largest[wave][col + e] = by_col[e];
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                by_col[e] = fmaxf(fmaxf(fmaxf(largest[0][col + e], largest[1][col + e]),
                                        fmaxf(largest[2][col + e], largest[3][col + e])), kLeastBlock);
                if (threadIdx.x < 16 && c0 + e < p.cols) p.scales_t[row_block * p.cols + c0 + e] = by_col[e] / kMostCode;
            }
        }
    }
    if (p.codes) {
        uint8_t* to = p.codes + c0;
        const uint64_t pitch = blocks_of(p.cols) * kWide;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= p.rows) continue;
            const float up = kMostCode / by_row[i];
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = raw[i].at(e) * up;
            *reinterpret_cast<u32x2*>(to + (r0 + i) * pitch) = codes8(v);
        }
    }
    if (p.codes_t) {
        uint8_t* to = p.codes_t + r0;
        const uint64_t pitch = blocks_of(p.rows) * kWide;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (c0 + e >= p.cols) continue;
            const float up = kMostCode / by_col[e];
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = raw[i].at(e) * up;
            *reinterpret_cast<u32x2*>(to + (c0 + e) * pitch) = codes8(v);
        }
    }
}

}  // namespace

template <class T, bool SQUARE>
static hipError_t launch_quantize_of(BlockParams p, hipStream_t s) {
    constexpr uint64_t MOST = 32768;  // rows of tiles to a launch
    const uint64_t high = blocks_of(p.rows);
    for (p.first = 0; p.first < high; p.first += MOST) {
        const uint64_t left = high - p.first;
        hipLaunchKernelGGL((quantize_kernel<T, SQUARE>), dim3((unsigned)blocks_of(p.cols), (unsigned)(left < MOST ? left : MOST)),
                           dim3(256), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_quantize(qsdp_dtype dtype, bool square, const BlockParams& p, hipStream_t s) {
    if (dtype == QSDP_F32) return square ? launch_quantize_of<F32, true>(p, s) : launch_quantize_of<F32, false>(p, s);
    if (dtype == QSDP_BF16) return square ? launch_quantize_of<BF16, true>(p, s) : launch_quantize_of<BF16, false>(p, s);
    return square ? launch_quantize_of<F16, true>(p, s) : launch_quantize_of<F16, false>(p, s);
}

}  // namespace qsdp_train
