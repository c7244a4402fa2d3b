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
// consecutive rows. The bytes bound it where there are many: 8192 x 8192 in bf16, 256 MiB read and written, 46.6 us or 5.8 TB/s (63 with
// largest values that neighbouring lanes find together, each with its quotients, and codes of columns stored eight at a time).
template <class T, bool SQUARE>
__global__ __launch_bounds__(256) void quantize_kernel(BlockParams p) {
    constexpr int ROW = 18;  // places of a row's parts: those of eight rows further on are in other banks
    __shared__ __attribute__((aligned(16))) float meet[SQUARE ? 16 : kWide * ROW + 16 * kWide];
    __shared__ __attribute__((aligned(16))) float ups[SQUARE ? 4 : 2 * kWide];
    __shared__ __attribute__((aligned(16))) uint8_t turned[kWide * kWide];
    const int col = threadIdx.x % 16 * 8, row = threadIdx.x / 16 * 8;
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
        most = fmaxf(reduce_block<256>(most, Max(), meet), kLeastBlock);
#pragma unroll
        for (int i = 0; i < 8; ++i) by_row[i] = by_col[i] = kMostCode / most;
        if (threadIdx.x == 0) {
            if (p.codes) p.scales[col_block * blocks_of(p.rows) + row_block] = most / kMostCode;
            if (p.codes_t) p.scales_t[row_block * blocks_of(p.cols) + col_block] = most / kMostCode;
        }
    } else {
        // The sixteen parts of a row's largest, and of a column's, meet in LDS; one thread has the quotients of a row or of a column.
        float* of_rows = meet;
        float* of_cols = meet + kWide * ROW;
#pragma unroll
        for (int i = 0; i < 8; ++i) of_rows[(row + i) * ROW + col / 8] = by_row[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) of_cols[row / 8 * kWide + col + e] = by_col[e];
        __syncthreads();
        const int in = threadIdx.x % kWide;
        const bool a_row = threadIdx.x < kWide;  // the same for a wave
        float most = kLeastBlock;
        if (a_row) {
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, of_rows[in * ROW + i]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, of_cols[i * kWide + in]);
        }
        ups[threadIdx.x] = kMostCode / most;
        const uint64_t r = row_block * kWide + in, c = col_block * kWide + in;
        if (a_row && p.codes && r < p.rows) p.scales[col_block * p.rows + r] = most / kMostCode;
        if (!a_row && p.codes_t && c < p.cols) p.scales_t[row_block * p.cols + c] = most / kMostCode;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) by_row[i] = ups[row + i], by_col[i] = ups[kWide + col + i];
    }
    if (p.codes) {
        uint8_t* to = p.codes + c0;
        const uint64_t pitch = blocks_of(p.cols) * kWide;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= p.rows) continue;
            const float up = by_row[i];
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = raw[i].at(e) * up;
            *reinterpret_cast<u32x2*>(to + (r0 + i) * pitch) = codes8(v);
        }
    }
    if (p.codes_t) {
        // Through LDS, so that a store writes whole lines: piece p of 16 rows of column c in place p ^ (c / 8), the columns past 64 with
        // their neighbours changed round, so that a wave's writes meet all banks.
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float up = by_col[e];
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = raw[i].at(e) * up;
            const int c = col + e, at = (c ^ c / 64) * (int)kWide + (row / 16 ^ c / 8 % 8) * 16 + row / 8 % 2 * 8;
            *reinterpret_cast<u32x2*>(turned + at) = codes8(v);
        }
        __syncthreads();
        const uint64_t pitch = blocks_of(p.rows) * kWide;
        uint8_t* to = p.codes_t + col_block * kWide * pitch + row_block * kWide;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = i * 32 + threadIdx.x / 8, piece = threadIdx.x % 8;
            if (col_block * kWide + c >= p.cols) continue;
            *reinterpret_cast<u32x4*>(to + c * pitch + piece * 16) =
                *reinterpret_cast<const u32x4*>(turned + (c ^ c / 64) * (int)kWide + (piece ^ c / 8 % 8) * 16);
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
