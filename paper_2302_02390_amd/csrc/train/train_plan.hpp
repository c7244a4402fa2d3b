// Which kernel a call of the training operators takes, by sizes alone (plain C++).
#pragma once
#include <cstdint>

namespace qsdp_train {

// ---- layer norm (train_norm.hip) -----------------------------------------------------------------------------------------
// Threads to a row, the fewest that hold it with 8 elements each (backward, which also holds its columns' sums) or 16 (forward).
// A wave to a row waits for nobody. SHORT: few rows of up to 2048 by four waves each, as nothing else fills the chip.
// STREAM: rows that no team holds, read again for each use.
enum class NormTeam { T64, T64_2, T128_2, T256_2, T512_2, T1024_2, T1024_4, SHORT, STREAM };

constexpr NormTeam choose_norm(uint64_t rows, uint64_t n) {
    if (n <= 512) return NormTeam::T64;
    if (n <= 2048 && rows <= 1024) return NormTeam::SHORT;
    if (n <= 1024) return NormTeam::T64_2;
    if (n <= 2048) return NormTeam::T128_2;
    if (n <= 4096) return NormTeam::T256_2;
    if (n <= 8192) return NormTeam::T512_2;
    if (n <= 16384) return NormTeam::T1024_2;
    if (n <= 32768) return NormTeam::T1024_4;
    return NormTeam::STREAM;
}

// T512_4: 32 elements to a thread of workgroups half as large, which have twice the registers each (4096 x 16384 in bf16 113 us; 152
// with 1024 threads of 16 elements, which spilled; 233 read again from memory).
enum class NormBackwardTeam { T64, T128, T256, T512, T1024, T512_4, STREAM };

constexpr NormBackwardTeam choose_norm_backward(uint64_t n) {
    if (n <= 512) return NormBackwardTeam::T64;
    if (n <= 1024) return NormBackwardTeam::T128;
    if (n <= 2048) return NormBackwardTeam::T256;
    if (n <= 4096) return NormBackwardTeam::T512;
    if (n <= 8192) return NormBackwardTeam::T1024;
    if (n <= 16384) return NormBackwardTeam::T512_4;
    return NormBackwardTeam::STREAM;
}

// Threads of a backward workgroup, and the rows that it has at once. (T512_4 has 512, for one row at a time.)
constexpr int kNormThreads = 1024;
constexpr uint64_t norm_rows_at_once(uint64_t n) {
    switch (choose_norm_backward(n)) {
        case NormBackwardTeam::T64: return kNormThreads / 64;
        case NormBackwardTeam::T128: return kNormThreads / 128;
        case NormBackwardTeam::T256: return kNormThreads / 256;
        case NormBackwardTeam::T512: return kNormThreads / 512;
        default: return 1;
    }
}

// Workgroups of the backward pass, each of which leaves one partial sum for the weight and one for the bias: what the chip runs
// at once. (Rows that no team holds: runs of rows, for every 2048 columns.)
constexpr uint64_t norm_workgroups(uint64_t rows, uint64_t n) {
    const uint64_t at_once = norm_rows_at_once(n), need = (rows + at_once - 1) / at_once;
    const uint64_t most = n <= 16384 ? 256 : 32;
    return need < most ? need : most;
}

// ---- products (train_product.hip) ------------------------------------------------------------------------------------------
constexpr uint64_t kFewRows = 16;

// Their kernels: workgroups that go through the columns, for rows whose codes fit into registers, or eight waves to 16 columns, or to 32,
// which share the rounding, where that leaves enough workgroups. Time by n x k of 16 rows, WIDE against TWO: 24 us for 38 at
// 50257 x 2048, 57 for 74 at 50257 x 4096, 10.1 for 9.7 at 16384 x 2048; TWO against ONE: 14.5 for 17.7 at 8192 x 4096, 7.7 for 7.1 at
// 4096 x 2048.
enum class FewKernel { ONE, TWO, WIDE };

constexpr FewKernel choose_few(uint64_t n, uint64_t k) {
    if (n >= 32768 && k <= 4096) return FewKernel::WIDE;
    return n >= 8192 ? FewKernel::TWO : FewKernel::ONE;
}

// Parts of a sum over `steps` blocks, each with at least `least` of them and none empty, that different workgroups add up and one more
// launch joins. Where `groups` workgroups fill the chip (256 or more) the parts cost more than they give.
constexpr uint64_t parts_of(uint64_t groups, uint64_t steps, uint64_t least) {
    const uint64_t by_steps = steps / least, by_groups = groups ? 448 / groups : 1;
    const uint64_t parts = by_steps < by_groups ? by_steps : by_groups;
    if (parts < 2) return 1;
    const uint64_t each = (steps + parts - 1) / parts;
    return (steps + each - 1) / each;
}

// Parts against none, by n x k: one row 11.3 us for 16.4 at 1024 x 16384, 10.1 for 11.3 at 2048 x 8192, 7.6 for 6.7 at 2048 x 4096; 16 rows
// 12.5 for 15.1 at 2048 x 8192, 19.0 for 16.0 at 4096 x 8192.
constexpr uint64_t choose_few_parts(uint64_t n, uint64_t k) {
    return choose_few(n, k) == FewKernel::ONE ? parts_of((n + 15) / 16, (k + 127) / 128, 24) : 1;
}

enum class ProductTile { T64, T128, T256, T64_4 };

// exact: results in binary32, whose operands take twice the registers in the 256-wide tile. T256 against T128, results in 16 bits:
// 134 us for 150 at 8192 x 8192 x 2048, 84 for 90 with k = 1024, 60 for 60 with 512; 61 for 57 at 6144 x 4096 x 2048, one pass and a half.
// T64 against T128: 13.8 us for 23 at 1000 x 1024 x 4096, 21.5 for 17.9 at 2048 x 2048 x 2048.
// T64_4: four steps in LDS, of which a compute unit has room for two tiles, instead of three: 7.5 us for 8.3 at 333 x 4093 x 1000, 12.0 for
// 13.1 at 1000 x 1024 x 4096, 12.1 for 10.5 at 1500 x 1500 x 1500 (576 tiles). Exact ones have two teams of waves instead.
// A tile counts whatever part of it the matrix fills: 17, 32 and 64 rows of 50257 x 2048 take tiles of 128, in 27.7, 28.0 and 30.1 us with
// their rounding (binary32: 37.8, 38.5, 40.4), for 24 us of 16 rows by the kernels of few rows.
constexpr ProductTile choose_tile(uint64_t m, uint64_t n, uint64_t k, bool exact) {
    const uint64_t of_128 = (m + 127) / 128 * ((n + 127) / 128), of_256 = (m + 255) / 256 * ((n + 255) / 256);
    // passes over the chip, whose compute units hold two of 128 or one of 256
    const uint64_t passes_128 = (of_128 + 511) / 512, passes_256 = (of_256 + 255) / 256;
    if (!exact && of_256 >= 224 && k >= 1024 && 9 * passes_256 <= 5 * passes_128) return ProductTile::T256;
    if (of_128 >= 224) return ProductTile::T128;
    return !exact && (m + 63) / 64 * ((n + 63) / 64) <= 512 ? ProductTile::T64_4 : ProductTile::T64;
}

// Parts against none, results in 16 bits: 13.4 us for 21.8 at 125 x 2048 x 8192, 26 for 40 at 768 x 768 x 16384, 11.3 for 12.5 at
// 125 x 2048 x 4096; of half the steps 9.4 for 7.9 at 125 x 2048 x 2048; of 256 tiles 17.8 for 13.2 at 1000 x 1024 x 4096.
constexpr uint64_t choose_parts(uint64_t m, uint64_t n, uint64_t k) {
    if (choose_tile(m, n, k, true) != ProductTile::T64) return 1;
    return parts_of((m + 63) / 64 * ((n + 63) / 64), (k + 127) / 128, 16);
}

}  // namespace qsdp_train
