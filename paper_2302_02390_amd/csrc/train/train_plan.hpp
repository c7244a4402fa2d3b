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

enum class NormBackwardTeam { T64, T128, T256, T512, T1024, T1024_2, STREAM };

constexpr NormBackwardTeam choose_norm_backward(uint64_t n) {
    if (n <= 512) return NormBackwardTeam::T64;
    if (n <= 1024) return NormBackwardTeam::T128;
    if (n <= 2048) return NormBackwardTeam::T256;
    if (n <= 4096) return NormBackwardTeam::T512;
    if (n <= 8192) return NormBackwardTeam::T1024;
    if (n <= 16384) return NormBackwardTeam::T1024_2;
    return NormBackwardTeam::STREAM;
}

// Threads of a backward workgroup, and the rows that it has at once.
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

// Groups of 16 columns to a workgroup: more of them share the rounding of the rows, fewer fill the chip.
constexpr int few_groups(uint64_t n) { return n >= 32768 ? 4 : n >= 8192 ? 2 : 1; }

enum class ProductTile { T64, T128, T256 };

// exact: results in binary32, whose operands take twice the registers in the 256-wide tile.
constexpr ProductTile choose_tile(uint64_t m, uint64_t n, uint64_t k, bool exact) {
    const uint64_t of_128 = (m + 127) / 128 * ((n + 127) / 128), of_256 = (m + 255) / 256 * ((n + 255) / 256);
    if (!exact && of_256 >= 224 && k >= 4096) return ProductTile::T256;
    return of_128 >= 224 ? ProductTile::T128 : ProductTile::T64;
}

}  // namespace qsdp_train
