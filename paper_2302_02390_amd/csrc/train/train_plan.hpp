// Which kernel a call of the training operators takes, by sizes alone (plain C++).
#pragma once
#include <cstdint>

namespace qsdp_train {

// ---- layer norm (train_norm.hip) -----------------------------------------------------------------------------------------
// Threads to a row, and groups of eight elements to a thread: a wave to a row as long as it holds one, as it then waits for
// nobody. WIDE: few short rows among four waves each, as nothing else fills the chip. STREAM: row read again for each use.
enum class NormTeam { W1, W2, W4, WIDE, T256, T1024, STREAM };

constexpr NormTeam choose_norm(uint64_t rows, uint64_t n) {
    if (n <= 512) return NormTeam::W1;
    if (n <= 2048 && rows <= 1024) return NormTeam::WIDE;
    if (n <= 1024) return NormTeam::W2;
    if (n <= 2048) return NormTeam::W4;
    if (n <= 8192) return NormTeam::T256;
    if (n <= 32768) return NormTeam::T1024;
    return NormTeam::STREAM;
}

enum class NormBackwardTeam { W1, W2, W4, T256, T512, STREAM };

constexpr NormBackwardTeam choose_norm_backward(uint64_t n) {
    if (n <= 512) return NormBackwardTeam::W1;
    if (n <= 1024) return NormBackwardTeam::W2;
    if (n <= 2048) return NormBackwardTeam::W4;
    if (n <= 8192) return NormBackwardTeam::T256;
    if (n <= 16384) return NormBackwardTeam::T512;
    return NormBackwardTeam::STREAM;
}

constexpr uint64_t kNormThreads = 512;  // of a backward workgroup

// Rows that a backward workgroup has at once.
constexpr uint64_t norm_rows_at_once(uint64_t n) {
    switch (choose_norm_backward(n)) {
        case NormBackwardTeam::W1: case NormBackwardTeam::W2: case NormBackwardTeam::W4: return kNormThreads / 64;
        case NormBackwardTeam::T256: return kNormThreads / 256;
        default: return 1;
    }
}

// Workgroups of the backward pass, each of which leaves one partial sum for the weight and one for the bias: one to a compute
// unit, and two where registers let two run. (Rows that no team holds: runs of rows, for every 2048 columns.)
constexpr uint64_t norm_workgroups(uint64_t rows, uint64_t n) {
    const uint64_t at_once = norm_rows_at_once(n), need = (rows + at_once - 1) / at_once;
    const uint64_t most = n <= 1024 ? 512 : n <= 16384 ? 256 : 32;
    return need < most ? need : most;
}

}  // namespace qsdp_train
