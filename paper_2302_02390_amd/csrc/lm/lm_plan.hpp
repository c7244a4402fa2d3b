// Which kernel a call of the operators on logits and on packed weights takes, by sizes and format alone (plain C++).
#pragma once
#include <cstdint>

namespace qsdp_lm {

// ---- rows of logits (lm_rows.hip) ----------------------------------------------------------------------------------------
// Threads and pieces of 16 bytes per thread by the row's length: the smallest team that holds it, as 64 registers to a lane keep
// a compute unit's 2048 threads; then with LDS, and the longest pass chunk by chunk.
enum class RowTeam { T128, T256, T512, T512_LDS, T1024, T1024_LDS, STREAM };

// Pieces in LDS: two workgroups of 1024 threads, four of 512, to a compute unit's 160 KB, with what else they use.
constexpr uint32_t held_pieces(int threads) { return threads == 1024 ? 4800 : 2240; }

// `per` elements to a piece; rows of 16-bit elements may have a lead of one.
constexpr uint64_t row_pieces(uint64_t n, uint64_t per) { return (n + per - 1 + (per == 8)) / per; }

// four: four workgroups of 512 threads to a compute unit, with LDS, rather than two of 1024 with registers alone: for what
// writes as much as it reads (distillation of 8192 rows of 50257 bf16 logits 332 / 354 us; sums alone of 4096 rows 75 / 70).
constexpr RowTeam choose_row(uint64_t pieces, bool four) {
    if (pieces <= 128 * 2) return RowTeam::T128;
    if (pieces <= 256 * 8) return RowTeam::T256;
    if (pieces <= 512 * 8) return RowTeam::T512;
    if (four && pieces <= 512 * 8 + held_pieces(512)) return RowTeam::T512_LDS;
    if (pieces <= 1024 * 8) return RowTeam::T1024;
    if (pieces <= 1024 * 8 + held_pieces(1024)) return RowTeam::T1024_LDS;
    return RowTeam::STREAM;
}

// Many rows with alternatives gain by four workgroups (4096 rows of 50257 bf16 logits, eight alternatives, 119 / 96 us), few lose
// (48 rows 10.5 / 12 us).
constexpr bool score_by_four(uint64_t rows, int top) { return top > 0 && rows >= 512; }

// ---- products (lm_linear.hip) ----------------------------------------------------------------------------------------------
constexpr int kStep = 128;  // codes

enum class Product {
    FEW_16_8, FEW_16_4, FEW_32_8, FEW_32_4,  // up to that many tokens, by so many waves
    TILE_64_TEAMS, TILE_64_DEEP, TILE_64, TILE_128, TILE_256
};

// Time of a product with tiles of tn x tm by the steps of 128 codes and the tiles that a compute unit gets: us of a step with
// one workgroup on the compute unit (it waits for its loads), of a step with all of them, and of a tile's start and end.
struct Cost {
    uint64_t tn, tm;
    double alone, packed, tile;
};
constexpr double cost_of(uint64_t m, uint64_t n, uint64_t k, const Cost& c) {
    const uint64_t tiles = (n + c.tn - 1) / c.tn * ((m + c.tm - 1) / c.tm), each = (tiles + 255) / 256;
    const double steps = (double)((k + kStep - 1) / kStep), step = c.packed * (double)each;
    return steps * (step > c.alone ? step : c.alone) + c.tile * (double)each;
}
// Measured on products of 8192 x 2048 x 8192, 4096^3, 2048^3, 512 x 8192 x 2048 and 512 x 2048 x 8192 (m x n x k), within a
// fifth of these sums: us with 256-, 128- and 64-wide tiles 142 / 171 / 251, 68 / 81 / 112, 36 / 18 / 19, 35 / 18 / 18 and
// 92 / 43 / 22.
constexpr Cost kCost256 = {256, 256, 1.43, 1.95, 11.0}, kCost128 = {128, 128, 0.66, 0.58, 3.5}, kCost64 = {64, 64, 0.30, 0.21, 1.3};

constexpr Product choose_small_tile(uint64_t m, uint64_t n, uint64_t k, uint64_t buckets) {
    // deeper where no more than two share a compute unit (512 x 2048 x 8192 32 / 22 us), else room for five (2048^3 22 / 19 us)
    const uint64_t tiles = (n + 63) / 64 * ((m + 63) / 64);
    // Several buckets and no more tiles than compute units: four teams to a tile where the steps are long enough to share (us without /
    // with, weights from memory: 125 x 2048 x 8192 in eight buckets 35.2 / 31.1, 512 x 2048 x 8192 35.0 / 30.1, 100 x 1024 x 4096 in
    // four 18.3 / 16.2, 125 x 2048 x 2048 in two 11.6 / 11.3; out of the caches 31.8 / 23.3, 31.9 / 24.0). With one bucket, whose sums
    // take nothing in between, teams lose as soon as the weights come from memory (125 x 2048 x 8192 23.1 / 27.4, 40 x 16384 x 2048
    // 11.9 / 13.3; out of the caches 19.8 / 18.9, 9.8 / 11.3).
    if (buckets > 1 && tiles <= 256 && k >= 2048) return Product::TILE_64_TEAMS;
    return tiles <= 512 ? Product::TILE_64_DEEP : Product::TILE_64;
}

constexpr Product choose_product(uint64_t m, uint64_t n, uint64_t k, uint64_t buckets) {
    // Few tokens: waves with loads of their own as long as the channels alone do not fill the chip, more of them to a channel where
    // there are fewer workgroups. Weights from memory, us by such waves / in tiles: 1 x 8192 x 2048 6.2 / 9.4, 16 x 2048 x 2048 4.5 / 8.5,
    // 32 x 4096 x 2048 5.9 / 9.8, 32 x 2048 x 8192 11 / 22; 16 x 50257 x 2048 29 / 24, 32 x 32768 x 2048 27 / 19. Between, the two cross
    // earlier for short channels (16 x 16384 x 2048 11.9 / 10.9, 32 x 16384 x 2048 14.5 / 11.7) and later for long ones (1 x 50257 x 8192
    // 82 / 106), which these limits leave out.
    const uint64_t groups = (n + 15) / 16;
    if (m <= 16 && groups <= 2048) return groups <= 512 ? Product::FEW_16_8 : Product::FEW_16_4;
    if (m <= 32 && groups <= 1024) return groups <= 256 ? Product::FEW_32_8 : Product::FEW_32_4;
    const double small = cost_of(m, n, k, kCost64), middle = cost_of(m, n, k, kCost128), large = cost_of(m, n, k, kCost256);
    if (buckets > 1)  // the largest tile has no registers for sums over buckets
        return small < middle ? choose_small_tile(m, n, k, buckets) : Product::TILE_128;
    if (small < middle && small < large) return choose_small_tile(m, n, k, buckets);
    return middle < large ? Product::TILE_128 : Product::TILE_256;
}

}  // namespace qsdp_lm
